"""Probabilities far below the largest one: a token of large score and value
zero among many of equal score, so that the output is what the small weights
hold.  Tolerances count the roundings: a weight's relative half step, with f16
elements at least 2^-40 of the largest weight, the scores' and sums' float32,
and the output's half step."""
import math

import pytest
import torch

import paper_2609_30950_amd as K
from tests import _attn as A
from tests._gpu import say

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,cache", [("f16", "same"), ("f16", "e4m3"), ("bf16", "same"), ("bf16", "e4m3")])
@pytest.mark.parametrize("drop", [15.5, 20.5, 25.25, 30.0, 35.0])
def test_step_one_large_score(dtype, cache, drop):
    lens, at, H, d, page, a = [33, 100, 2000, 131], [0, 50, 1999, 130], 2, 64, 16, 4.0
    B, t = len(lens), A.TYPES[dtype]
    held = [-(-n // page) for n in lens]
    cfg = K.AttnConfig(K.Pages(B, page, sum(held), max(held)), 2 * H, H, d, dtype=dtype, cache=cache, scale=math.log(2.0))
    g = torch.Generator(device="cuda").manual_seed(1)
    tables, slots, first = [], [], 0
    for n, h in zip(lens, held):
        tables.append(list(range(first, first + h)) + [0] * (max(held) - h))
        slots += [first * page + i for i in range(n)]
        first += h
    k = torch.zeros(len(slots), H, d, device="cuda", dtype=t)
    v = (16 * (0.5 + torch.rand(len(slots), H, d, device="cuda", generator=g))).to(t)
    start = [sum(lens[:b]) for b in range(B)]
    for b in range(B):
        k[start[b] + at[b], :, 0] = a            # its score: a * q = drop octaves
        v[start[b] + at[b]] = 0.0
    kc, vc = K.new_attn_caches(cfg)
    scale = {}
    if cache == "e4m3":
        scale = dict(k_scale=torch.ones(H, device="cuda"), v_scale=torch.full((H,), 256.0, device="cuda"))
        v = v.float().to(A.E4M3).to(t)
        K.kda_attn_append(cfg, k, v, torch.tensor(slots, **I32), kc, vc)
    else:
        v = v * 256
        K.kda_attn_append(cfg, k, v, torch.tensor(slots, **I32), kc, vc)
    q = torch.zeros(B, 2 * H, d, device="cuda", dtype=t)
    q[:, :, 0] = drop / a
    o = torch.empty(B, 2 * H, d, device="cuda", dtype=t)
    lse = torch.empty(B, 2 * H, device="cuda")
    K.kda_attn_step(cfg, q, kc, vc, torch.tensor(tables, **I32), torch.tensor(lens, **I32), o,
                    K.new_attn_workspace(cfg), lse=lse, **scale)
    torch.cuda.synchronize()
    u, floor, small = A.half_step(t), 2.0 ** -40 if dtype == "f16" else 0.0, 2.0 ** -drop
    worst = [0.0, 0.0]
    for b, n in enumerate(lens):
        vals = v[start[b]:start[b] + n].double().repeat_interleave(2, 1) * (256.0 if cache == "e4m3" else 1.0)
        e = 4 * 2.0 ** -24 * drop + 2.0 ** -21 + n * 2.0 ** -24 / 8
        total = 1.0 + (n - 1) * small
        want = vals.sum(0) * small / total
        bound = vals.sum(0) / total * (small * (u + 2.2 * e) + floor) * (1 + u) + want * u * 1.01 + 2.0 ** -25
        worst[0] = max(worst[0], float(((o[b].double() - want).abs() / bound).max()))
        wl = drop * math.log(2.0) + math.log1p((n - 1) * small)
        worst[1] = max(worst[1], float((lse[b].double() - wl).abs().max()) / (1.1 * e + wl * 2.0 ** -22))
    say(f"small weights 2^-{drop} {dtype} {cache}: {worst[0]:.3f} of the output bound, {worst[1]:.3f} of the log sum's")
    assert worst[0] <= 1.0 and worst[1] <= 1.0
