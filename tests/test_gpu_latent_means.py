"""Latent step: weighted means of the latent vectors that are small or large
beside f16's range, against their exact values.  The tolerance counts the
probabilities' half step, the pair that the mean enters the last product as,
the output's half step and the float32 sums."""
import pytest
import torch

import paper_2609_30950_amd as K
from tests import _attn as A
from tests._gpu import say

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,size,weight", [("bf16", 2.0 ** -30, 2.0 ** 20), ("bf16", 2.0 ** -12, 2.0 ** 10),
                                               ("bf16", 2.0 ** 40, 2.0 ** -40), ("f16", 2.0 ** -22, 2.0 ** 14),
                                               ("f16", 2.0 ** -14, 2.0 ** 12), ("f16", 2.0 ** 14, 2.0 ** -8)])
@pytest.mark.parametrize("lens", [[40, 1], [3000, 130, 0, 900]], ids=str)
def test_step_means_of_any_size(dtype, size, weight, lens):
    H, dn, dr, dc, page = 17, 64, 32, 256, 64
    B, t = len(lens), A.TYPES[dtype]
    held = [-(-n // page) for n in lens]
    cfg = K.LatentConfig(K.Pages(B, page, sum(held), max(held)), H=H, d_n=dn, d_r=dr, d_c=dc, d_v=dn, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    tables, first = [], 0
    for h in held:
        tables.append(list(range(first, first + h)) + [0] * (max(held) - h))
        first += h
    cache = K.new_latent_cache(cfg)
    # the same scores everywhere; one token in sixteen has a latent vector
    live = (torch.arange(cfg.pages.n_pages * page, device="cuda") % 16 == 0).reshape(-1, page, 1)
    cache[..., :dc] = (size * live * (1 + torch.rand(cfg.pages.n_pages, page, dc, device="cuda", generator=g))).to(t)
    w_uk = torch.zeros(H, dn, dc, device="cuda", dtype=t)
    w_uv = (weight * torch.randn(H, dn, dc, device="cuda", generator=g) / 16).to(t)
    q_n, q_r = (torch.zeros(B, H, x, device="cuda", dtype=t) for x in (dn, dr))
    o = torch.empty(B, H, dn, device="cuda", dtype=t)
    K.kda_latent_step(cfg, q_n, q_r, w_uk, w_uv, cache, torch.tensor(tables, **I32), torch.tensor(lens, **I32), o,
                      K.new_latent_workspace(cfg))
    torch.cuda.synchronize()
    u, eps, worst = A.half_step(t), 2.0 ** -24, 0.0
    pair, floor = (u * u, 0.0) if dtype == "bf16" else (u * u, 2.0 ** -36)
    for b, n in enumerate(lens):
        if n == 0:
            assert not bool(o[b].any())
            continue
        c = cache.flatten(0, 1)[int(tables[b][0]) * page:][:n, :dc].double().mean(0)
        w = w_uv.double()
        want, size_w = w @ c, w.abs() @ c
        bound = size_w * (u + pair + (dc + n / 8 + 24) * eps) * (1 + u) + w.abs().sum(2) * floor + want.abs() * u * 1.01
        bound = bound + (2.0 ** -25 if dtype == "f16" else 0.0)
        worst = max(worst, float(((o[b].double() - want).abs() / bound).max()))
    say(f"latent means {size} {dtype} {lens}: {worst:.3f} of the bound")
    assert worst <= 1.0
