"""cqsa_cache_weigh against the float64 oracle.

The bound: a weight exp(s - LSE) is off relatively by what its exponent is off, whose fp32
sum of d exact products and whose steps (times the scale, minus LSE, in powers of two) round at
most d + 8 times at the size of the sum of |q k| or LSE, and by some units of the exponential; a sum of n
positive terms adds n half steps, and W one.
"""
import math

import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import bounded as ob
from oracle import cache4 as o4
from tests.gpu_util import need_gpu, say
from tests.op_util import DT, WEIGH_LOOPS, Case, normal, starts

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -24


def attended(case, cache, batch, q, causal, scale=0.0):
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), math.nan, device="cuda")
    cq.cqsa_cache_attend(cache, batch, q, torch.empty_like(q), lse, causal=causal, scale=scale)
    return lse


def check(case, q, lse, W, new, counts, causal, scale, prior, decay, packed, first=0, oracle=ob.weigh):
    """Every sequence's weights against the oracle; what lies behind its tokens is untouched."""
    torch.cuda.synchronize()
    d, G = case.d, q.shape[2] // case.H
    Wc, lc, qc = W.cpu().double().numpy(), lse.cpu().double().numpy(), q.cpu().double().numpy()
    at, worst = first, 0.0
    for b, (n, m) in enumerate(zip(case.lens, new)):
        rows = slice(at, at + m) if packed else slice(0, m)
        bb = 0 if packed else b
        page, tok = case.slots(b, 0, n)
        k, _ = o4.read(case.data, case.page, case.H, d, page, tok)
        there = (page >= 0) & (page < case.n_pages)
        old = None if prior is None else prior[b].cpu().double().numpy()
        c = m if counts is None else min(max(int(counts[b]), 0), m)
        want, big = oracle(qc[bb, rows], k, lc[bb][:, rows].T, there, n, c, causal, scale, old, decay)
        got = Wc[b, :, :n]
        bound = want * HALF * ((d + 8) * big + c * G + 16) + 1e-36
        err = np.abs(got - want)
        assert np.isfinite(got).all() and (err <= bound).all(), (b, err.max(), (err / bound).max())
        worst = max(worst, (err / bound).max() if err.size else 0.0)
        assert (Wc[b, :, n:] == 7.0).all()
        at += m
    return worst


def run(case, Hq, new, dtype, causal=True, counts=None, decay=1.0, with_prior=True, packed=False, scale=0.0,
        max_len=0, first=0, spare=3, in_place=False, oracle=ob.weigh):
    g = case.g
    T = case.table.shape[1] * case.page + spare
    shape = (1, first + sum(new) + 2, Hq, case.d) if packed else (len(new), new[0], Hq, case.d)
    q = normal(g, shape, dtype).cuda()
    cache = case.cache()
    batch = case.batch(q_start=starts(new, first) if packed else None, max_len=max_len, max_q=max(max(new), 1) if packed else 0)
    lse = attended(case, cache, batch, q, causal, scale)
    prior = torch.from_numpy(g.random((len(new), case.H, T), dtype=np.float32)).cuda() if with_prior else None
    if prior is not None:  # what the rows' own tokens and those behind hold is not read
        for b, (n, m) in enumerate(zip(case.lens, new)):
            prior[b, :, max(0, n - m):] = math.nan
    W = torch.full((len(new), case.H, T), 7.0, device="cuda")
    keep = prior
    if in_place:
        keep = prior.clone()
        for b, n in enumerate(case.lens):
            prior[b, :, n:] = 7.0
        W = prior
    cnt = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_weigh(cache, batch, q, lse, W, prior=prior, decay=decay, counts=cnt, causal=causal, scale=scale)
    return check(case, q, lse, W, new, counts, causal, scale or 1 / math.sqrt(case.d), keep, decay, packed, first, oracle)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_step(d, dtype):
    need_gpu()
    say("weigh step", d, dtype)
    case = Case(d, [131, 1, 0, 64, 33], 2, d, 64)
    case.fill_tokens()
    run(case, 6, [1] * 5, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [32, 96, 128, 224, 256])
@pytest.mark.parametrize("n,G", [(17, 1), (40, 4), (9, 8)])
def test_chunk(d, dtype, n, G):
    """More rows than a tile's, causal, beginning before position 0 in the shorter sequences."""
    need_gpu()
    say("weigh chunk", d, dtype, n, G)
    case = Case(d + n, [150, 20, 5], 2, d, 32)
    case.fill_tokens()
    run(case, 2 * G, [n] * 3, dtype, decay=0.75)


def any_tokens(case, power=122):
    """Fills the pool with random codes, whose powers are near 2^(power - 127)."""
    case.data = case.g.integers(0, 256, case.data.shape, dtype=np.uint8)
    tiles = case.data.reshape(case.n_pages, -1, 34 * case.d)
    tiles[..., 32 * case.d:] = power + tiles[..., 32 * case.d:] % 3


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,n,L,page", [(32, 8500, 150, 256), (96, 8200, 97, 32), (128, 8193, 140, 64), (160, 1700, 81, 128),
                                        (256, 1801, 70, 64), (256, 900, 70, 32)])
def test_long_contexts(d, n, L, page, dtype):
    """Many rows over contexts for which work groups have more waves, with splits of the rows."""
    need_gpu()
    say("weigh long", d, n, L, dtype)
    case = Case(n + d, [n, n // 3, L // 2], 1, d, page)
    any_tokens(case)
    case.table[0, 1] = -1
    run(case, 4, [L] * 3, dtype, counts=[L, L - 7, L], decay=0.5, oracle=ob.weigh_rows if n > 1000 else ob.weigh)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,n,L", [(32, 32771, 35), (64, 16390, 40), (64, 16384, 33)])
def test_one_long_context(d, n, L, dtype):
    """A single sequence, for whose narrow heads work groups have more waves only then."""
    need_gpu()
    say("weigh one long", d, n, L, dtype)
    case = Case(n + d, [n], 1, d, 128)
    any_tokens(case)
    case.table[0, 1] = -1
    run(case, 4, [L], dtype, decay=0.5, oracle=ob.weigh_rows)


@pytest.mark.parametrize("d", [192, 224, 256])
@pytest.mark.parametrize("n,G", [(33, 1), (16, 4), (11, 4), (13, 5)])
def test_rows_held_for_wide_heads(d, n, G):
    """33 to 65 fp32 rows over more tokens than a work group's, and fewer."""
    need_gpu()
    say("weigh wide", d, n, G)
    case = Case(d + n, [1100, 515, 40, 5], 2, d, 64)
    any_tokens(case)
    run(case, 2 * G, [n] * 4, "f32", decay=0.75)


@pytest.mark.parametrize("rows", [1, 2, 4, 5, 16, 17, 32, 33, 63, 64, 65, 127, 128, 129, 192, 257])
def test_row_counts(rows):
    """Around the borders between the kernels, and a kernel's own steps."""
    need_gpu()
    say("weigh rows", rows)
    case = Case(rows, [700, 260, 90], 2, 64, 64)
    any_tokens(case)
    run(case, 2, [rows] * 3, "bf16", causal=False, oracle=ob.weigh_rows)
    run(case, 2, [rows] * 3, "f16", causal=False, oracle=ob.weigh_rows)


def test_more_sequences_and_heads_than_one_dimension_takes():
    """2^21 work groups and more; every sequence has the same tokens and queries."""
    need_gpu()
    say("weigh many heads")
    for L, G in ((1, 1), (20, 2)):
        B, H = 32768, 65
        case = Case(L, [40], H, 32, 64, extra_columns=0)
        any_tokens(case)
        cache = case.cache()
        table = torch.from_numpy(case.table).cuda().expand(B, -1)
        batch = cq.CacheBatch(table.contiguous(), torch.full((B,), 40, dtype=torch.int32, device="cuda"))
        q = normal(case.g, (1, L, H * G, 32), "bf16").cuda().expand(B, -1, -1, -1)
        lse = torch.zeros(B, H * G, L, device="cuda")
        W = torch.full((B, H, 64), 7.0, device="cuda")
        cq.cqsa_cache_weigh(cache, batch, q, lse, W)
        one = torch.full((1, H, 64), 7.0, device="cuda")
        cq.cqsa_cache_weigh(cache, case.batch(), q[:1].contiguous(), lse[:1].contiguous(), one)
        check(case, q[:1], lse[:1], one, [L], None, True, 32 ** -0.5, None, 1.0, False, oracle=ob.weigh_rows)
        # one sequence's rows may be added in another order
        assert torch.allclose(W, one.expand(B, -1, -1), rtol=2.0 ** -18)


@pytest.mark.parametrize("page", [32, 64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_pages_and_masks(page, causal):
    need_gpu()
    say("weigh pages", page, causal)
    case = Case(page, [300, 257, 31, 2], 3, 64, page)
    case.fill_tokens()
    run(case, 3, [4] * 4, "bf16", causal=causal, scale=0.3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_packed_rows(dtype):
    """Packed rows between rows that no sequence has, some sequences without rows."""
    need_gpu()
    say("weigh packed", dtype)
    case = Case(5, [70, 40, 90, 3, 0], 2, 96, 32)
    case.fill_tokens()
    run(case, 4, [7, 0, 33, 5, 2], dtype, packed=True, first=3, decay=0.5)


def test_counts():
    need_gpu()
    say("weigh counts")
    case = Case(6, [50, 40, 45, 60, 33], 2, 64, 32)
    case.fill_tokens()
    run(case, 4, [6] * 5, "f16", counts=[6, 0, 3, 99, -4])


def test_in_place_and_without_prior():
    need_gpu()
    say("weigh in place")
    case = Case(7, [90, 33], 2, 128, 64)
    case.fill_tokens()
    run(case, 4, [3, 3], "bf16", decay=0.9, in_place=True)
    run(case, 4, [3, 3], "bf16", with_prior=False, decay=0.9)
    run(case, 4, [3, 3], "bf16", decay=0.0)
    cache, batch = case.cache(), case.batch()
    q = normal(case.g, (2, 3, 4, 128), "bf16").cuda()
    lse = attended(case, cache, batch, q, True)
    a = torch.full((2, 2, case.table.shape[1] * 64), 7.0, device="cuda")
    b = a.clone()
    cq.cqsa_cache_weigh(cache, batch, q, lse, a)
    cq.cqsa_cache_weigh(cache, batch, q, lse, b, prior=torch.full_like(b, math.nan), decay=0.0)
    assert torch.equal(a, b)  # nothing of a prior that counts for nothing


def test_pages_that_hold_nothing():
    need_gpu()
    say("weigh holes")
    case = Case(8, [200, 100], 2, 64, 32)
    case.fill_tokens()
    case.table[0, 2] = -1
    case.table[0, 4] = 10 ** 6
    case.table[1, 0] = -7
    run(case, 2, [2, 2], "bf16")


def test_nan_tokens_and_rows():
    """A NaN token makes the rows that see it add nothing; the other rows' sums are as without it."""
    need_gpu()
    say("weigh nan")
    case = Case(9, [64], 1, 64, 32)
    case.fill_tokens()
    page, tok = case.slots(0, 61, 1)
    k = np.full((1, 1, 64), np.nan)
    o4.write(case.data, 32, k, k, page, tok)
    g = case.g
    q = normal(g, (1, 8, 2, 64), "bf16").cuda()
    q[0, 1, 0, 5] = math.nan
    cache, batch = case.cache(), case.batch()
    lse = attended(case, cache, batch, q, True)
    assert torch.isnan(lse[0, :, 5:]).all() and torch.isnan(lse[0, 0, 1])
    W = torch.zeros(1, 1, 96, device="cuda")
    cq.cqsa_cache_weigh(cache, batch, q, lse, W)
    q = torch.nan_to_num(q)
    rows = lse.clone()
    torch.cuda.synchronize()
    k, _ = o4.read(case.data, 32, 1, 64, *case.slots(0, 0, 64))
    want, big = ob.weigh(q.cpu().double().numpy()[0], np.nan_to_num(k), rows.cpu().double().numpy()[0].T,
                         np.ones(64, bool), 64, 8, True, 1 / 8.0, None, 1.0)
    got = W.cpu().double().numpy()[0, :, :64]
    assert (np.abs(got - want) <= want * HALF * (72 * big + 32) + 1e-36).all()
    assert got[0, 61] == 0


def test_infinite_lse():
    need_gpu()
    say("weigh infinite lse")
    case = Case(10, [40], 1, 32, 32)
    case.fill_tokens()
    q = normal(case.g, (1, 3, 1, 32), "bf16").cuda()
    lse = torch.tensor([[[-math.inf, math.inf, math.nan]]], device="cuda")
    W = torch.full((1, 1, 96), 5.0, device="cuda")
    cq.cqsa_cache_weigh(case.cache(), case.batch(), q, lse, W)
    assert (W[0, 0, :40] == 0).all() and (W[0, 0, 40:] == 5).all()


def test_sums_are_the_rows():
    """The weights of one row's tokens sum to 1, over many splits of a long context too."""
    need_gpu()
    say("weigh sums")
    for B, n, L in ((1, 70001, 1), (2, 5003, 3), (1, 2500, 700)):
        case = Case(n, [n] * B, 2, 64, 256)
        case.data = case.g.integers(0, 256, case.data.shape, dtype=np.uint8)
        tiles = case.data.reshape(case.n_pages, -1, 34 * 64)
        tiles[..., 32 * 64:] = 125 + tiles[..., 32 * 64:] % 3
        q = normal(case.g, (B, L, 4, 64), "bf16").cuda()
        cache, batch = case.cache(), case.batch()
        lse = attended(case, cache, batch, q, False)
        W = torch.zeros(B, 2, case.table.shape[1] * 256, device="cuda")
        cq.cqsa_cache_weigh(cache, batch, q, lse, W, causal=False)
        # the errors of LSE and of the weights, 64 products' and 2^10 units at most
        assert torch.allclose(W.double().sum(-1), torch.full((B, 2), 2.0 * L, dtype=torch.float64, device="cuda"), rtol=1e-4)


@pytest.mark.parametrize("d,dtype,G,max_len", [(32, "bf16", 8, 2 ** 20), (64, "f16", 1, 2 ** 20), (64, "f32", 8, 2 ** 20),
                                               (128, "bf16", 8, 2 ** 19), (160, "f32", 8, 2 ** 19)])
def test_sums_of_many_rows(d, dtype, G, max_len):
    """Weights of 131072 rows that are all alike: the roundings of one long sum, in which equal terms are
    added, would all go the same way (2e-5 of the sum and more).

    Half steps of a sum: 2 LSE for the exponent (LSE in powers of two, rounded twice), 2 for the exponential,
    4 and 32 for the rows that a lane adds before it compensates what it loses, 2 for that sum itself, 2 for
    the lanes' and W's."""
    need_gpu()
    say("weigh many rows", d, dtype, G, max_len)
    H, rows, n, page = 8, 131072, 300, 256
    pages = torch.full((1, max_len // page), -1, dtype=torch.int32, device="cuda")
    pages[0, :2] = torch.tensor([1, 0])
    cache = cq.Cache4(2, H, d, page_size=page)  # zeros: every score is 0
    # the bound on the lengths gives work groups enough that the rows are not split
    batch = cq.CacheBatch(pages, torch.tensor([n], dtype=torch.int32, device="cuda"), max_len=max_len)
    q = torch.zeros(1, rows // G, H * G, d, dtype=DT[dtype], device="cuda")
    assert cq.cqsa_cache_weigh_workspace(cache, batch, q) is None
    lse = (1.1 + 0.37 * torch.arange(H, device="cuda")).repeat_interleave(G)[None, :, None].expand(1, H * G, rows // G).contiguous()
    W = torch.full((1, H, max_len), 7.0, device="cuda")
    cq.cqsa_cache_weigh(cache, batch, q, lse, W, causal=False)
    e = lse[0, ::G, 0].double()
    want = (rows * torch.exp(-e))[:, None]
    off = ((W[0, :, :n].double() - want) / want).abs()
    assert (off <= ((2 * e + 44) * HALF)[:, None]).all(), off.max().item()
    assert (W[0, :, n:] == 7).all()


def test_sums_past_the_last_number():
    """Weights that are infinite, by an LSE that no attention left, give an infinite sum, not a NaN."""
    need_gpu()
    say("weigh infinite sums")
    H, d, rows, max_len = 2, 32, 4096, 2 ** 16
    pages = torch.full((1, max_len // 256), -1, dtype=torch.int32, device="cuda")
    pages[0, 0] = 0
    cache = cq.Cache4(1, H, d, page_size=256)
    batch = cq.CacheBatch(pages, torch.tensor([90], dtype=torch.int32, device="cuda"), max_len=max_len)
    q = torch.zeros(1, rows, H, d, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros(1, H, rows, device="cuda")
    lse[0, 1, 100] = -100.0
    W = torch.zeros(1, H, max_len, device="cuda")
    cq.cqsa_cache_weigh(cache, batch, q, lse, W, causal=False)
    assert (W[0, 0, :90] == rows).all() and (W[0, 1, :90] == math.inf).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,H,G,L,d,dtype,n", WEIGH_LOOPS)
def test_waves_of_several_tiles(B, H, G, L, d, dtype, n, in_place):
    """Keys, pages and prior of a wave's next tile are read while it works on one: every token's own prior, and
    a page that holds nothing among them.  (tests/test_operator_lanes.py: that these calls' waves go through several.)"""
    need_gpu()
    say("weigh loops", B, H, G, L, d, dtype, n, in_place)
    page, scale = 64, 1 / math.sqrt(d)
    lens = [n if b == 0 else int(n * (b * 0.6180339887 % 1.0)) for b in range(B)]
    g = torch.Generator("cuda").manual_seed(n + d)
    need = [-(-x // page) for x in lens]
    pages = torch.full((B, need[0]), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(sum(need), generator=g, device="cuda").int()
    for b, m in enumerate(need):
        pages[b, :m] = order[sum(need[:b]):sum(need[:b]) + m]
    pages[0, need[0] // 2] = -1
    data = torch.randint(0, 256, (sum(need), cq.cqsa_cache_page_bytes(page, H, d)), generator=g, device="cuda", dtype=torch.uint8)
    data.view(sum(need), -1, 34 * d)[..., 32 * d:] = 121 + data.view(sum(need), -1, 34 * d)[..., 32 * d:] % 3
    cache = cq.Cache4(sum(need), H, d, page_size=page, data=data)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    batch = cq.CacheBatch(pages, lengths, max_len=n)
    q = torch.randn(B, L, H * G, d, generator=g, device="cuda").to(DT[dtype])
    lse = attended(None, cache, batch, q, True)
    prior = torch.rand(B, H, n, generator=g, device="cuda") + 0.5
    before = prior.double()
    W = prior if in_place else torch.full_like(prior, 7.0)
    cq.cqsa_cache_weigh(cache, batch, q, lse, W, prior=prior, decay=0.75)
    t = torch.arange(n, device="cuda")
    for b, m in enumerate(lens):
        k, v = torch.empty(2, 1, max(m, 1), H, d, device="cuda").unbind(0)
        cq.cqsa_cache_read(cache, cq.CacheBatch(pages[b:b + 1], lengths[b:b + 1]), k, v)
        del v
        kk = k[0, max(m, 1) - m:].double().transpose(0, 1).contiguous()
        qq = q[b].double().view(L, H, G, d).permute(1, 3, 0, 2).reshape(H, d, L * G).contiguous()
        l = lse[b].double().view(H, G, L).transpose(1, 2).reshape(H, 1, L * G)
        row = torch.arange(L, device="cuda").repeat_interleave(G)
        seen = (t[:m, None] <= m - L + row) & (pages[b, t[:m] // page] >= 0)[:, None]
        w = torch.exp((torch.matmul(kk, qq) * scale - l).masked_fill(~seen, -math.inf)).sum(-1)
        size = torch.matmul(kk.abs(), qq.abs()) * scale
        big = torch.maximum(size, l.abs().expand_as(size)).masked_fill(~seen, 0.0).amax(-1)
        old = max(0, m - L)
        w[:, :old] += 0.75 * before[b, :, :old]
        off = (W[b, :, :m].double() - w).abs()
        assert (off <= w * HALF * ((d + 8) * big + L * G + 16) + 1e-36).all(), (b, off.max().item())
        behind = before[b, :, m:].float() if in_place else torch.full_like(W[b, :, m:], 7.0)
        assert torch.equal(W[b, :, m:], behind)


def test_strided_tensors_and_another_stream():
    need_gpu()
    say("weigh strides")
    case = Case(11, [77, 50], 2, 64, 32)
    case.fill_tokens()
    both = normal(case.g, (2, 3, 9, 64), "bf16").cuda()
    q = both[:, :, 3:7]
    store = torch.full((2, 5, 200), 7.0, device="cuda")
    W = store[:, 1:3, 10:170]
    cache, batch = case.cache(), case.batch()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lse = attended(case, cache, batch, q, True)
        cq.cqsa_cache_weigh(cache, batch, q, lse, W)
    torch.cuda.current_stream().wait_stream(side)
    check(case, q, lse, W, [3, 3], None, True, 0.125, None, 1.0, False)
    store[:, 1:3, 10:170] = 7.0
    assert (store == 7).all()


def test_weights_far_apart():
    """Weights whose elements lie past 2^31."""
    need_gpu()
    say("weigh far")
    case = Case(13, [90, 70], 2, 64, 32)
    case.fill_tokens()
    cache, batch = case.cache(), case.batch()
    T, far = case.table.shape[1] * 32, 2 ** 31 + 12345
    for L in (2, 100):
        q = normal(case.g, (2, L, 2, 64), "bf16").cuda()
        lse = attended(case, cache, batch, q, True)
        store = torch.empty(far + 10 ** 6, device="cuda")
        W = store.as_strided((2, 2, T), (far, T + 3, 1))
        W.fill_(7.0)
        cq.cqsa_cache_weigh(cache, batch, q, lse, W)
        check(case, q, lse, W, [L, L], None, True, 0.125, None, 1.0, False)
        cq.cqsa_cache_weigh(cache, batch, q, lse, W, prior=W, decay=0.5)
        assert torch.isfinite(W).all()


def test_python_refusals():
    need_gpu()
    case = Case(14, [40, 30], 2, 64, 32)
    cache, batch = case.cache(), case.batch()
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse, W = torch.zeros(2, 4, 3, device="cuda"), torch.zeros(2, 2, 96, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(cache=cache, batch=batch, Q=q, LSE=lse, W=W)
    for bad in (dict(Q=q.cpu()), dict(Q=q[0]), dict(LSE=lse[:, :2]), dict(LSE=lse.double()), dict(W=W.half()), dict(W=W[0]),
                dict(W=W.transpose(1, 2)), dict(prior=W.cpu()), dict(counts=n[:1]), dict(counts=n.long()),
                dict(workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            cq.cqsa_cache_weigh(**{**ok, **bad})
    for bad in (dict(W=W[..., :50]), dict(W=W[:1].expand(2, -1, -1)), dict(prior=W[..., 1:].as_strided((2, 2, 96), (96, 96, 1))),
                dict(decay=2.0), dict(scale=math.inf)):
        with pytest.raises(cq.CqsaError):
            cq.cqsa_cache_weigh(**{**ok, **bad})
    cq.cqsa_cache_weigh(**ok)


def test_missing_arguments_are_named():
    need_gpu()
    case = Case(14, [40, 30], 2, 64, 32)
    cache, batch = case.cache(), case.batch()
    q = torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16, device="cuda")
    lse, W = torch.zeros(2, 4, 3, device="cuda"), torch.zeros(2, 2, 96, device="cuda")
    with pytest.raises(ValueError, match="LSE must"):
        cq.cqsa_cache_weigh(cache, batch, q, None, W)
    with pytest.raises(ValueError, match="W must"):
        cq.cqsa_cache_weigh(cache, batch, q, lse, None)
    with pytest.raises(ValueError, match="W must"):
        cq.cqsa_cache_evict(cache, batch, None, torch.zeros(2, dtype=torch.int32, device="cuda"), 10)


def test_same_bits_again_and_captured():
    """Two calls give the same bits, and so does every replay of a captured one."""
    need_gpu()
    say("weigh captured")
    for lens, L in (([3000, 100], 1), ([900], 300)):
        case = Case(12, lens, 2, 128, 64)
        case.fill_tokens()
        q = normal(case.g, (len(lens), L, 8, 128), "bf16").cuda()
        cache, batch = case.cache(), case.batch()
        lse = attended(case, cache, batch, q, True)
        prior = torch.rand(len(lens), 2, case.table.shape[1] * 64, device="cuda")
        W = torch.zeros_like(prior)
        space = cq.cqsa_cache_weigh_workspace(cache, batch, q)
        call = lambda: cq.cqsa_cache_weigh(cache, batch, q, lse, W, prior=prior, decay=0.5, workspace=space)
        call()
        first = W.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for i in range(4):
            W.fill_(float(i))
            if space is not None:
                space.fill_(255 - i)
            graph.replay()
            torch.cuda.synchronize()
            for b, n in enumerate(lens):
                assert torch.equal(W[b, :, :n], first[b, :, :n])
