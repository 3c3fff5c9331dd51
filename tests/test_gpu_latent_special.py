"""Latent attention with NaN and infinities in weights, latent vectors, shared
key parts and queries: they reach the outputs that the definition gives them,
and no others."""
import pytest
import torch

import paper_2609_30950_amd as K
from tests import _attn as A
from tests.test_gpu_latent import _check, _prefill, _step, _world

pytestmark = pytest.mark.gpu
INF = float("inf")
SHAPES = [([150, 0, 70], [150, 3, 30]), ([3000, 40], [5, 2])]   # in one part, and cut into several


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sizes", [(64, 32, 256), (128, 64, 512), (64, 64, 512), (128, 32, 256)], ids=str)
@pytest.mark.parametrize("lens,rows", SHAPES, ids=str)
def test_prompts_value_weights(dtype, sizes, lens, rows):
    """A value channel whose weights are not finite is NaN, where the row has
    tokens; the other channels stay as they were."""
    s = _world(41, lens, 5, *sizes, dtype=dtype, rows=rows)
    clean, dn = _prefill(s), sizes[0]
    assert bool(clean.isfinite().all())
    want = clean.clone()
    bad = [(0, 0, 0, float("nan")), (1, 37, 3, INF), (1, 38, sizes[2] - 1, -INF), (3, 31, 100, float("nan")),
           (4, dn - 1, 7, float("nan"))]
    for h, d, j, x in bad:
        s["w_uv"][h, d, j] = x
        for b in range(len(lens)):
            if lens[b]:
                want[int(s["cu"][b]):int(s["cu"][b + 1]), h, d] = float("nan")
    o = _prefill(s)
    assert torch.equal(o.isnan(), want.isnan()) and torch.equal(o.nan_to_num(3.0), want.nan_to_num(3.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompts_value_weights_of_many_heads(dtype):
    s = _world(42, [300, 20], 131, 64, 32, 256, dtype=dtype, rows=[200, 20])
    clean = _prefill(s)
    g = torch.Generator(device="cuda").manual_seed(1)
    bad = torch.rand(131, 64, device="cuda", generator=g) < 0.1
    s["w_uv"][..., 200] = torch.where(bad, float("nan"), s["w_uv"][..., 200])
    o = _prefill(s)
    assert torch.equal(o.isnan(), bad.expand_as(o)) and torch.equal(o[:, ~bad], clean[:, ~bad])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B", [3, 70])
def test_step_value_weights(dtype, B):
    """As in prompts: the channel is NaN, and zero where there are no tokens."""
    lens = [(0, 1, 90, 700)[b % 4] for b in range(B)]
    s = _world(48, lens, 20, 64, 32, 256, dtype=dtype)
    clean = _step(s)
    s["w_uv"][3, 17, 100] = s["w_uv"][19, 63, 255] = float("nan")
    some = torch.tensor(lens, device="cuda") > 0
    want = clean.clone()
    want[some, 3, 17] = want[some, 19, 63] = float("nan")
    o = _step(s)
    assert torch.equal(o.isnan(), want.isnan()) and torch.equal(o.nan_to_num(3.0), want.nan_to_num(3.0))
    assert not bool(o[~some].any())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("value", [INF, -INF, float("nan")])
@pytest.mark.parametrize("lens,rows,at", [([150], [150], 100), ([3000], [5], 2997)], ids=str)
def test_latent_vectors(dtype, value, lens, rows, at):
    s = _world(43, lens, 3, 64, 32, 256, dtype=dtype, rows=rows)
    clean = _prefill(s)
    s["cache"][int(s["tables"][0, at // 64]), at % 64, 9] = value
    s["w_uk"][1, 5, 9] = s["w_uv"][2, 8, 9] = 0.0
    first = at - (lens[0] - rows[0])                    # the first row that sees the token
    o = _prefill(s)
    assert bool(o[first:].isnan().all()) and bool(o[:first].isfinite().all())
    assert torch.equal(o[:first, 0], clean[:first, 0])
    assert bool(_step(dict(s, q_n=s["q_n"][-1:], q_r=s["q_r"][-1:])).isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("value", [INF, -INF])
def test_shared_key_parts(dtype, value):
    """A score of +inf leaves NaN, one of -inf takes the token out."""
    n, at = 150, 100
    s = _world(44, [n], 4, 64, 32, 256, dtype=dtype, rows=[n])
    pid, off = int(s["tables"][0, at // 64]), at % 64
    s["cache"][pid, off, 256 + 11] = value
    up = s["q_r"][:, :, 11].sign() * (1.0 if value > 0 else -1.0) > 0
    seen = torch.arange(n, device="cuda") >= at
    o = _prefill(s)
    assert torch.equal(o.isnan(), (up & seen[:, None])[..., None].expand_as(o))
    rows, pos = A.request_rows(s["cache"], s["tables"][0].tolist(), n, 64, s["cfg"].pages.n_pages)
    keep = pos != at
    want, bound = A.latent(s["q_n"], s["q_r"], rows[keep], pos[keep], torch.arange(n, device="cuda"), s["w_uk"],
                           s["w_uv"], 96 ** -0.5, 2.0 ** -11, True)
    u = A.half_step(s["cfg"]._t)
    bound = bound * (1 + u) + want.abs() * u * 1.01 + float(torch.finfo(s["cfg"]._t).tiny)
    assert bool(((o.double() - want).abs() <= bound)[~o.isnan()].all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("part", ["q_n", "q_r"])
def test_queries(dtype, part):
    s = _world(45, [200], 4, 64, 32, 256, dtype=dtype, rows=[200])
    clean, were = _prefill(s), s[part].clone()
    s[part][150, 2, 5] = INF                            # scores of both signs
    s[part][151, 1, 5] = float("nan")
    o = _prefill(s)
    assert bool(o[150, 2].isnan().all()) and bool(o[151, 1].isnan().all())
    # rows that share a wave may take another reference of their weights: the
    # bounds hold, not the bits
    o[150, 2], o[151, 1] = clean[150, 2], clean[151, 1]
    s[part].copy_(were)
    _check(s, o, True)


def test_large_finite_numbers_are_cut():
    """bf16 elements past f16's range, in latent vectors, keys and queries: cut
    to 65504, never infinite."""
    s = _world(46, [100], 2, 64, 32, 256, rows=[100])
    s["cache"][int(s["tables"][0, 0]), 3] = 1e30
    s["q_n"][40, 1, 3] = -1e30
    assert bool(_prefill(s).isfinite().all())


def test_clean_inputs_check():
    s = _world(47, [150, 0, 70], 5, 64, 32, 256, rows=[150, 0, 30])
    _check(s, _prefill(s), True)
