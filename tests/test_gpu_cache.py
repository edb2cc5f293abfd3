"""Writing the 4-bit cache and reading it back on the GPU, against oracle.cache4.

Every comparison is exact: the format leaves no choice of rounding.
"""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import cache4 as o4
from paper_2604_20819_amd import synth
from tests.gpu_util import need_gpu, say
from tests.op_util import DT, Case, normal, starts

pytestmark = pytest.mark.gpu


def written(case, lens, new, rows_k, rows_v):
    """The oracle's pool after the call's rows (float64, per sequence) are written."""
    data = case.data.copy()
    for b, (n, m) in enumerate(zip(lens, new)):
        p, t = case.slots(b, n - m, m)
        o4.write(data, case.page, rows_k[b], rows_v[b], p, t)
    return data


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,H,page,lens,new", [
    (32, 1, 32, (1,), 1), (64, 2, 64, (5, 64, 65, 200), 1), (128, 8, 64, (33, 97, 128), 7),
    (96, 3, 32, (300, 31), 31), (160, 1, 128, (129,), 129), (192, 2, 256, (70, 300), 70),
    (224, 1, 64, (64,), 64), (256, 2, 32, (100, 40), 40)])
def test_write_and_read(dtype, d, H, page, lens, new):
    need_gpu()
    case = Case(d + H, lens, H, d, page)
    B = len(lens)
    k, v = (normal(case.g, (B, new, H, d), dtype) * 3 for _ in range(2))
    k[..., 3] *= 50
    say("write", dtype, d, H, page, lens, new)
    cache, batch = case.cache(), case.batch()
    cq.cqsa_cache_write(cache, batch, k.cuda(), v.cuda())
    want = written(case, lens, [new] * B, synth.as_f64(k), synth.as_f64(v))
    assert np.array_equal(cache.data.cpu().numpy(), want)
    ko, vo = (torch.full_like(k, 9.0, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, batch, ko, vo)
    for b, n in enumerate(lens):
        p, t = case.slots(b, n - new, new)
        rk, rv = o4.read(want, page, H, d, p, t)
        for got, ref in ((ko[b], rk), (vo[b], rv)):
            assert torch.equal(got.cpu(), torch.from_numpy(ref).to(DT[dtype]))


def test_read_in_every_type():
    """What one type wrote reads the same in the others, fp16 rounded."""
    need_gpu()
    case = Case(4, (77,), 2, 64, 32)
    case.fill_tokens(gain=1e-4)
    cache, batch = case.cache(), case.batch()
    p, t = case.slots(0, 0, 77)
    want = o4.read(case.data, 32, 2, 64, p, t)
    for dtype in DT.values():
        out = [torch.empty((1, 77, 2, 64), dtype=dtype, device="cuda") for _ in range(2)]
        cq.cqsa_cache_read(cache, batch, *out)
        for got, ref in zip(out, want):
            assert torch.equal(got[0].cpu(), torch.from_numpy(ref).to(dtype))


def test_every_code_and_border():
    """Values at and beside every border between codes, at many powers; zeros, the smallest and
    largest magnitudes, infinities and NaN."""
    need_gpu()
    d = 64
    at = np.concatenate([np.arange(0, 8, 0.125), [6.99, 7.0, 7.01, 5.0, 0.25, 0.75]])
    rows = []
    for power in (-100, -20, -3, 0, 1, 15, 90):
        x = np.concatenate([at, np.nextafter(np.float32(at), np.float32(9)), np.nextafter(np.float32(at), np.float32(0))])
        x = np.concatenate([x, -x]).astype(np.float32) * np.float32(2.0 ** power)
        x = np.resize(x, (-(-len(x) // d) * d,))
        rows.append(x.reshape(-1, d))
    x = np.concatenate(rows)
    special = np.zeros((6, d), np.float32)
    special[1, :] = -0.0
    special[2, 5], special[2, 40] = np.inf, 1.0
    special[3, 7] = np.nan
    special[4, :32], special[4, 32:] = 1e-42, 2.0 ** -126
    special[5, :32], special[5, 32:] = 3.4e38, -1.6e38
    x = torch.from_numpy(np.concatenate([x, special]))[None, :, None]
    n = x.shape[1]
    case = Case(1, (n,), 1, d, 64)
    cache, batch = case.cache(), case.batch()
    y = x.flip(1).contiguous()
    cq.cqsa_cache_write(cache, batch, x.cuda(), y.cuda())
    want = written(case, [n], [n], synth.as_f64(x), synth.as_f64(y))
    assert np.array_equal(cache.data.cpu().numpy(), want)
    ko, vo = torch.empty_like(x, device="cuda"), torch.empty_like(x, device="cuda")
    cq.cqsa_cache_read(cache, batch, ko, vo)
    p, t = case.slots(0, 0, n)
    rk, rv = o4.read(want, 64, 1, d, p, t)
    for got, ref in ((ko, rk), (vo, rv)):
        assert np.array_equal(got[0].cpu().double().numpy(), ref, equal_nan=True)


@pytest.mark.parametrize("page", [32, 128])
def test_packed_rows(page):
    """Ragged rows, some sequences with none, rows that no sequence has, and rows before
    position 0."""
    need_gpu()
    lens, new, first = (70, 0, 33, 3, 128), (65, 0, 1, 9, 128), 4
    H, d = 2, 64
    case = Case(7, lens, H, d, page)
    T = first + sum(new) + 5
    k, v = (normal(case.g, (1, T, H, d), "bf16") for _ in range(2))
    cache = case.cache()
    batch = case.batch(q_start=starts(new, first), max_q=128)
    cq.cqsa_cache_write(cache, batch, k.cuda(), v.cuda())
    off = first + np.concatenate([[0], np.cumsum(new)])
    rows = [[synth.as_f64(x)[0, off[b]:off[b + 1]] for b in range(len(lens))] for x in (k, v)]
    want = written(case, lens, new, *rows)
    assert np.array_equal(cache.data.cpu().numpy(), want)
    ko, vo = (torch.full((1, T, H, d), 9.0, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, batch, ko, vo)
    for got, w in ((ko, 0), (vo, 1)):
        got = got[0].cpu().double().numpy()
        assert (got[:first] == 9).all() and (got[off[-1]:] == 9).all()
        for b, (n, m) in enumerate(zip(lens, new)):
            p, t = case.slots(b, n - m, m)
            assert np.array_equal(got[off[b]:off[b + 1]], o4.read(want, page, H, d, p, t)[w])


def test_values_out_of_range_are_clamped():
    """Pages outside the pool, lengths and starts outside their range: nothing is written
    outside the rows' places, and the rest is as documented."""
    need_gpu()
    H, d, page = 1, 32, 32
    case = Case(3, (64, 96, 20), H, d, page)
    case.table[0, 1], case.table[1, 0] = case.n_pages, -5
    k, v = (normal(case.g, (3, 64, H, d), "f32") for _ in range(2))
    lens = [64, 2 ** 31 - 1, -7]
    cache = case.cache()
    batch = case.batch(lens=lens, max_len=96)
    cq.cqsa_cache_write(cache, batch, k.cuda(), v.cuda())
    real = [64, 96, 0]
    want = written(case, real, [64] * 3, synth.as_f64(k), synth.as_f64(v))
    assert np.array_equal(cache.data.cpu().numpy(), want)
    ko, vo = (torch.full_like(k, 9.0, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, batch, ko, vo)
    for b, n in enumerate(real):
        p, t = case.slots(b, n - 64, 64)
        assert np.array_equal(ko[b].cpu().double().numpy(), o4.read(want, page, H, d, p, t)[0])
    # starts that fall, and leave the tensor
    T = 10
    q_start = torch.tensor([-3, 4, 2, 99], dtype=torch.int32, device="cuda")
    x = normal(case.g, (1, T, H, d), "f32")
    cache = case.cache()
    cq.cqsa_cache_write(cache, case.batch(lens=[64, 96, 20], q_start=q_start, max_q=5), x.cuda(), x.cuda())
    data = case.data.copy()
    # sequence 0: rows 0 .. 3; 1: none; 2: rows 2 .. 9, of which max_q lets 5
    for b, lo, m, n in ((0, 0, 4, 64), (2, 2, 5, 20)):
        p, t = case.slots(b, n - m, m)
        r = synth.as_f64(x)[0, lo:lo + m]
        o4.write(data, page, r, r, p, t)
    assert np.array_equal(cache.data.cpu().numpy(), data)


def test_strided_rows():
    need_gpu()
    B, L, H, d = 2, 40, 2, 64
    case = Case(5, (40, 77), H, d, 64)
    qkv = normal(case.g, (B, L, 8, d), "f16")
    w = qkv.cuda()
    cache, batch = case.cache(), case.batch()
    cq.cqsa_cache_write(cache, batch, w[:, :, 4:6], w[:, :, 6:8])
    want = written(case, case.lens, [L] * B, synth.as_f64(qkv[:, :, 4:6].contiguous()),
                   synth.as_f64(qkv[:, :, 6:8].contiguous()))
    assert np.array_equal(cache.data.cpu().numpy(), want)
    out = torch.zeros((B, L, 8, d), dtype=torch.float16, device="cuda")
    cq.cqsa_cache_read(cache, batch, out[:, :, 1:3], out[:, :, 5:7])
    k, v = (torch.empty((B, L, H, d), dtype=torch.float16, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, batch, k, v)
    assert torch.equal(out[:, :, 1:3], k) and torch.equal(out[:, :, 5:7], v)
    assert not out[:, :, [0, 3, 4, 7]].any()


def test_pages_beyond_four_gigabytes():
    need_gpu()
    H, d, page = 8, 128, 256
    per = cq.cqsa_cache_page_bytes(page, H, d)
    n_pages = (9 << 29) // per  # 4.5 GiB
    data = torch.zeros((n_pages, per), dtype=torch.uint8, device="cuda")
    cache = cq.Cache4(n_pages, H, d, page_size=page, data=data)
    table = torch.tensor([[n_pages - 1, 0]], dtype=torch.int32, device="cuda")
    batch = cq.CacheBatch(table, torch.tensor([300], dtype=torch.int32, device="cuda"))
    g = np.random.Generator(np.random.PCG64(8))
    k, v = (normal(g, (1, 300, H, d), "bf16") for _ in range(2))
    cq.cqsa_cache_write(cache, batch, k.cuda(), v.cuda())
    ko, vo = (torch.empty_like(k, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, batch, ko, vo)
    for got, x in ((ko, k), (vo, v)):
        want = o4.values(*o4.quantise(synth.as_f64(x)))
        assert np.array_equal(got.cpu().double().numpy(), want)
    assert not data[1:n_pages - 1].any()


def test_captured_step():
    """One token a sequence written under a graph, replayed for new rows."""
    need_gpu()
    H, d = 2, 64
    case = Case(2, (33, 64, 1), H, d, 32)
    cache, batch = case.cache(), case.batch()
    k, v = (torch.zeros((3, 1, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cq.cqsa_cache_write(cache, batch, k, v)
        cq.cqsa_cache_read(cache, batch, ko, vo)
    for _ in range(3):
        a, b = (normal(case.g, (3, 1, H, d), "bf16") for _ in range(2))
        k.copy_(a)
        v.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for got, x in ((ko, a), (vo, b)):
            assert np.array_equal(got.cpu().double().numpy(), o4.values(*o4.quantise(synth.as_f64(x))))


def test_sequences_that_share_a_page():
    """Two sequences write neighbouring tokens of one page, and of one tile, in one call."""
    need_gpu()
    H, d, page = 3, 96, 64
    case = Case(6, (5, 41), H, d, page)
    case.table[1] = case.table[0]
    new = (5, 36)  # tokens 0 .. 4 and 5 .. 40
    k, v = (normal(case.g, (1, sum(new), H, d), "bf16") for _ in range(2))
    cache = case.cache()
    cq.cqsa_cache_write(cache, case.batch(q_start=starts(new), max_q=max(new)), k.cuda(), v.cuda())
    p, t = case.slots(1, 0, 41)
    o4.write(case.data, page, synth.as_f64(k)[0], synth.as_f64(v)[0], p, t)
    assert np.array_equal(cache.data.cpu().numpy(), case.data)
