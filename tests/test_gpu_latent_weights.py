"""Latent attention with probabilities far below the largest one: a token of
large score and latent vector zero among many of equal score, so that the
output is what the small weights hold.  Tolerances count the roundings: a
weight's relative half step and a floor relative to the largest weight (step
with f16 elements 2^-40, prompts 2^-36), the scores' and sums' float32, in
prompts the values' f16, and the output's half step."""
import math

import pytest
import torch

import paper_2609_30950_amd as K
from tests import _attn as A
from tests._gpu import say

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def _world(lens, at, drop, dtype, rows, dn=64):
    """Token at[b] of request b scores `drop` octaves above the others."""
    H, dr, dc, page, a = 3, 32, 256, 16, 4.0
    B, t = len(lens), A.TYPES[dtype]
    held = [-(-n // page) for n in lens]
    cfg = K.LatentConfig(K.Pages(B, page, sum(held), max(held)), H=H, d_n=dn, d_r=dr, d_c=dc, d_v=dn, dtype=dtype,
                         scale=math.log(2.0))
    g = torch.Generator(device="cuda").manual_seed(2)
    cache = K.new_latent_cache(cfg)
    tables, first, vals = [], 0, []
    for b, (n, h) in enumerate(zip(lens, held)):
        tables.append(list(range(first, first + h)) + [0] * (max(held) - h))
        rowsb = cache[first:first + h].flatten(0, 1)
        rowsb[:n, 1] = (0.5 + torch.rand(n, device="cuda", generator=g)).to(t)
        rowsb[at[b]] = 0.0
        rowsb[at[b], dc] = a
        vals.append(rowsb[:n, 1].double())
        first += h
    w_uk = torch.zeros(H, dn, dc, device="cuda", dtype=t)
    w_uv = torch.zeros(H, dn, dc, device="cuda", dtype=t)
    w_uv[:, :, 1] = 2.0 ** 12
    n = sum(rows)
    q_n = torch.zeros(n, H, dn, device="cuda", dtype=t)
    q_r = torch.zeros(n, H, dr, device="cuda", dtype=t)
    q_r[..., 0] = drop / a
    return dict(cfg=cfg, cache=cache, tables=torch.tensor(tables, **I32), lens=torch.tensor(lens, **I32), q_n=q_n,
                q_r=q_r, w_uk=w_uk, w_uv=w_uv, vals=vals, o=torch.empty(n, H, dn, device="cuda", dtype=t))


def _share(o, vals, at, seen, drop, dtype, floor, roundings):
    """Worst share of the bound of rows that see the first `seen` tokens."""
    u, small = A.half_step(A.TYPES[dtype]), 2.0 ** -drop
    total, biggest = (1.0 + (seen - 1) * small, 1.0) if at < seen else (float(seen), 1.0)
    if at >= seen:
        small = 1.0
    e = 4 * 2.0 ** -24 * drop + 2.0 ** -21 + seen * 2.0 ** -24 / 8
    sum_v = float(vals[:seen].sum()) * 2.0 ** 12
    want = sum_v * small / total
    bound = sum_v / total * (small * (roundings + 2.2 * e) + floor * biggest) * (1 + u) + want * u * 1.01 + 2.0 ** -25
    return float((o.double() - want).abs().max()) / bound


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("drop", [15.5, 20.5, 25.25, 30.0, 35.0])
def test_step_one_large_score(dtype, drop):
    lens, at = [33, 100, 2000, 131], [0, 50, 1999, 130]
    s = _world(lens, at, drop, dtype, [1] * len(lens))
    K.kda_latent_step(s["cfg"], s["q_n"], s["q_r"], s["w_uk"], s["w_uv"], s["cache"], s["tables"], s["lens"], s["o"],
                      K.new_latent_workspace(s["cfg"]))
    torch.cuda.synchronize()
    u = A.half_step(A.TYPES[dtype])
    floor = 2.0 ** -40 if dtype == "f16" else 0.0
    worst = max(_share(s["o"][b], s["vals"][b], at[b], n, drop, dtype, floor, u + u * u) for b, n in enumerate(lens))
    say(f"small weights 2^-{drop} latent step {dtype}: {worst:.3f} of the bound")
    assert worst <= 1.0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dn", [64, 128])
@pytest.mark.parametrize("drop", [3.75, 7.5, 15.5, 20.5, 25.25, 30.0])
def test_prompts_one_large_score(dtype, dn, drop):
    """Chains in one block, in parts, and the large score first, amid and last."""
    for lens, at, rows in (([700, 90, 33], [0, 60, 32], [130, 90, 33]), ([5000], [0], [3]), ([5000], [2222], [3]),
                           ([1500], [1499], [2])):
        s = _world(lens, at, drop, dtype, rows, dn)
        cu = [sum(rows[:b]) for b in range(len(rows) + 1)]
        K.kda_latent_prefill(s["cfg"], sum(lens), s["q_n"], s["q_r"], torch.tensor(cu, **I32), s["w_uk"], s["w_uv"],
                             s["cache"], s["tables"], s["lens"], s["o"],
                             K.new_latent_prefill_workspace(s["cfg"], sum(lens)))
        torch.cuda.synchronize()
        worst = 0.0
        for b, n in enumerate(lens):
            for i in range(rows[b]):
                seen = n - rows[b] + i + 1
                worst = max(worst, _share(s["o"][cu[b] + i], s["vals"][b], at[b], seen, drop, dtype, 2.0 ** -36,
                                          2 * 2.0 ** -11 * (1 + 2.0 ** -11)))
        say(f"small weights 2^-{drop} prompts {dtype} d={dn} {lens}: {worst:.3f} of the bound")
        assert worst <= 1.0
