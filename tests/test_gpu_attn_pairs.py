"""The attention step rounds its result once: the probabilities enter the second
product as pairs, whose rounding (the square of a half step, with f16 elements
at least 2^-40 of the largest) is far below the output's."""
import pytest
import torch

from tests import _attn as A
from tests import test_gpu_attn as G
from tests._gpu import say

pytestmark = G.pytestmark


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("f16", "same"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_step_rounds_once(dtype, cache, d):
    lens = [1, 33, 150, 2000, 700]
    s = G._world(61, 5, 8, 2, d, 32, lens, dtype, cache)
    o, lse = G._step(s)
    cfg, worst, off, size_all = s["cfg"], 0.0, 0.0, 0.0
    kc, vc = s["kc"].double(), s["vc"].double()
    if s["scale"]:
        kc = kc * s["scale"]["k_scale"].double()[:, None, None]
        vc = vc * s["scale"]["v_scale"].double()[:, None, None, None]
    u = A.half_step(cfg._t)
    for b, n in enumerate(lens):
        k, v = A.request_kv(kc, vc, s["tables"][b].tolist(), n, 32, cfg.pages.n_pages)
        want, _, size, width = A.attend(s["q"][b], k, v, A.sqrt_scale(d))
        e = (A.score_error(d, width.cuda()) + n * 2.0 ** -24 / 8)[:, None]
        floor = n * 2.0 ** -40 * v.abs().amax() if dtype == "f16" else 0.0
        bound = size * (u * u + 2.2 * e) * (1 + u) + floor + want.abs() * u * 1.01 + 2.0 ** -25
        err = (o[b].double() - want).abs()
        worst = max(worst, float((err / bound).max()))
        off, size_all = off + float(err.square().sum()), size_all + float(want.square().sum())
    say(f"attn d={d} {dtype} {cache}: {worst:.3f} of the bound, norm {(off / size_all) ** 0.5 / u:.3f} half steps")
    assert worst <= 1.0
