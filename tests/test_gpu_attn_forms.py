"""Forms of the attention layers' kernels that only larger calls take: plans
that move many pages, appends whose single rows take all heads in turn, the
join of wide heads for many requests, the join of the latent step with eight
requests a block, and prompts of many query tiles over long contexts."""
import random

import pytest
import torch

import paper_2609_30950_amd as K
from tests import _attn as A
from tests import test_gpu_attn as G
from tests import test_gpu_latent as L

pytestmark = G.pytestmark


@pytest.mark.parametrize("B,page,max_pages,most,spare,n_slots", [(200, 16, 400, 900, 3000, 1000),
                                                                 (1025, 32, 100, 200, 9000, 60000)])
def test_plan_of_many_pages(B, page, max_pages, most, spare, n_slots):
    rng = random.Random(B)
    lens, new, n_pages, free, tables = G._random_step(rng, B, page, max_pages, most, spare)
    back = sum(-(-n // page) for n, x in zip(lens, new) if x < 0)
    assert back > (1024 if n_slots <= 1024 else 4096)          # more than one turn of the moves
    want = A.plan(page, max_pages, n_pages, lens, new, spare, free, tables, n_slots)
    for alias in (False, True):
        got = G._run_plan(K.Pages(B, page, n_pages, max_pages), lens, new, spare, free, tables, n_slots, alias)
        assert got == want, [k for k in want if want[k] != got[k]]


def test_plan_waiting_requests_behind_rows_past_the_slots():
    # request 1's rows pass the slots: 2 and 4 wait behind them (0, nothing
    # changes for them), 3 ends; before them request 0 waits (1)
    page, lens, new = 16, [5, 3, 20, 17, 0], [0, 9, 0, -1, 0]
    tables = [[0, -1], [1, -1], [2, 3], [4, 5], [-1, -1]]
    free = [6, 7, -1, -1, -1, -1, -1, -1]
    got = G._run_plan(K.Pages(5, page, 8, 2), lens, new, 2, free, tables, 4)
    assert got["ok"] == [1, 0, 0, 1, 0] and got["lens"] == [5, 3, 20, 0, 0] and got["cu"] == [0, 0, 9, 9, 9, 9]
    assert got["tables"] == tables and got["slots"] == [-1] * 4 and got["free"][:4] == [6, 7, 4, 5]


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("f16", "e4m3")])
@pytest.mark.parametrize("n,H,d,page", [(4099, 5, 128, 16), (2500, 7, 128, 256), (1100, 8, 256, 64)])
def test_append_of_many_rows(dtype, cache, n, H, d, page):
    # a run of tokens that begins and ends amid an octet, then single rows in
    # any order, padding rows among both
    assert n * H * d // 8 >= 1 << 18
    g = torch.Generator(device="cuda").manual_seed(n)
    n_pages = n // page + 3
    cfg = K.AttnConfig(K.Pages(1, page, n_pages, 1), H, H, d, dtype=dtype, cache=cache)
    kv = torch.randn(n, 2 * H, d, device="cuda", generator=g).to(A.TYPES[dtype])
    run, total = 2 * n // 3, n_pages * page
    slots = torch.empty(n, **G.I32)
    slots[:run] = torch.arange(3, 3 + run, **G.I32)
    slots[run:] = (3 + run + torch.randperm(total - 3 - run, device="cuda", generator=g)[:n - run]).to(torch.int32)
    slots[100], slots[run + 5], slots[n - 1] = -1, -9, total
    kc, vc = K.new_attn_caches(cfg)
    raw = torch.uint8 if cache == "e4m3" else torch.int16
    for x in (kc, vc):
        x.view(raw).copy_(torch.randint(0, 100, x.shape, device="cuda", generator=g).to(raw))
    before = [x.clone() for x in (kc, vc)]
    scale = {}
    k, v = kv[:, :H], kv[:, H:]
    if cache == "e4m3":
        scale = dict(k_scale=0.01 + torch.rand(H, device="cuda", generator=g),
                     v_scale=torch.linspace(0.01, 0.02, H).cuda())
    K.kda_attn_append(cfg, k, v, slots, kc, vc, **scale)
    if cache == "e4m3":
        quant = lambda x, s: (x.float() / s[:, None]).clamp(-448, 448).to(A.E4M3)  # noqa: E731
        k, v = quant(k, scale["k_scale"]), quant(v, scale["v_scale"])
    live = (slots >= 0) & (slots < total)
    to = slots[live].long()
    wk, wv = (x.view(raw) for x in before)
    wk[to // page, :, to % page] = k[live].contiguous().view(raw)
    wv[to // page, :, to % page // 8, :, to % 8] = v[live].contiguous().view(raw)
    assert torch.equal(kc.view(raw), wk) and torch.equal(vc.view(raw), wv)


@pytest.mark.parametrize("dtype,cache", [("bf16", "same"), ("f16", "same"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("d", [128, 256])
def test_join_of_wide_heads_for_many_requests(dtype, cache, d):
    # 20 x 32 heads: a block joins a whole head; requests of one part, of several and of many
    rng = random.Random(d)
    lens = [rng.choice([0, 1, 40, 129, 700, 2000]) for _ in range(20)]
    lens[3], lens[11] = 9000, 0
    s = G._world(51, 20, 32, 4, d, 64, lens, dtype, cache)
    G._check_step(s, *G._step(s), only=[0, 3, 4, 11, 19] + rng.sample(range(20), 6))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,H,sizes", [(57, 32, (128, 64, 512)), (64, 32, (64, 32, 256)), (60, 33, (64, 64, 512)),
                                       (63, 40, (128, 32, 256))], ids=str)
def test_latent_join_of_eight_requests_a_block(dtype, B, H, sizes):
    # 256 to 511 blocks of a head and eight requests, the last of them not full
    rng = random.Random(B)
    lens = [rng.choice([0, 1, 30, 300, 1200]) for _ in range(B)]
    lens[5] = 6000
    s = L._world(52, lens, H, *sizes, dtype=dtype)
    L._check(s, L._step(s), False, only=[0, 5, 7, 8, B - 2, B - 1] + rng.sample(range(B), 6))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("sizes", L.SIZES, ids=str)
def test_prompts_of_many_tiles_over_long_contexts(dtype, sizes):
    # 128 heads, five query tiles and more: one team of waves a block
    s = L._world(53, [1500, 20, 700], 128, *sizes, dtype=dtype, rows=[500, 20, 129], page=32)
    s["tables"][0, 20] = -1
    L._check(s, L._prefill(s), True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_prompts_of_many_requests_over_long_contexts(dtype):
    rng = random.Random(9)
    lens = [rng.choice([300, 900, 1400]) for _ in range(40)]
    rows = [rng.choice([1, 2, 60]) for _ in lens]
    s = L._world(54, lens, 16, 128, 64, 512, dtype=dtype, rows=rows)
    L._check(s, L._prefill(s), True, only=[0, 1, 20, 38, 39])
