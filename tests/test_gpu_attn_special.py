"""The attention step over tokens whose values or keys are not finite: as the
definition has it, in the heads and channels concerned alone."""
import pytest
import torch

from tests import test_gpu_attn as G

pytestmark = G.pytestmark
INF = float("inf")


def _place(s, b, t):
    page = s["cfg"].pages.page
    return int(s["tables"][b, t // page]), t % page


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_values(dtype, d):
    s = G._world(71, 3, 8, 2, d, 32, [150, 1, 3000], dtype)
    clean, lse = G._step(s)
    want = clean.clone()
    for b, t, hk, c, x in ((0, 7, 0, 3, INF), (0, 149, 1, d - 1, -INF), (1, 0, 0, 5, INF), (2, 1234, 1, 17, float("nan")),
                           (2, 40, 0, 0, -INF), (2, 2999, 0, 9, INF), (2, 30, 0, 9, -INF)):
        pid, off = _place(s, b, t)
        s["vc"][pid, hk, off // 8, c, off % 8] = x
        want[b, 4 * hk:4 * hk + 4, c] = x
    want[2, 0:4, 9] = float("nan")                      # one of each sign
    o, lse2 = G._step(s)
    assert torch.equal(lse, lse2)
    assert torch.equal(o.nan_to_num(7.0, 1e4, -1e4), want.nan_to_num(7.0, 1e4, -1e4))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_keys(dtype):
    s = G._world(72, 2, 8, 2, 128, 32, [150, 700], dtype)
    clean, lse = G._step(s)
    pid, off = _place(s, 1, 333)
    s["kc"][pid, 1, off, 20] = INF
    o, lse2 = G._step(s)
    up = s["q"][1, 4:, 20] > 0                          # +inf: NaN; -inf: the token has no weight
    assert bool(o[1, 4:][up].isnan().all()) and bool(o[1, 4:][~up].isfinite().all())
    assert torch.equal(o[0], clean[0]) and torch.equal(o[1, :4], clean[1, :4])
    assert torch.equal(lse2[1, :4], lse[1, :4]) and bool(lse2[1, 4:][~up].isfinite().all())
