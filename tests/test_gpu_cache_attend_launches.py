"""Attention over the 4-bit cache on the GPU through launches that are named and checked:
work groups of 8, 12 and 16 waves, and two groups of 16 rows a wave.  Bounds as in
tests/test_gpu_cache_attend.py."""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import cache4 as o4
from paper_2604_20819_amd import synth
from tests.gpu_util import need_gpu, say
from tests.op_util import Case, normal
from tests.test_gpu_cache_attend import bounded, held, reference, run

pytestmark = pytest.mark.gpu


def launch(case, q, kind="few", **kw):
    return cq.cqsa_cache_attend_launch(case.cache(), bounded(case, kind, **kw), q.cuda())


WAVES = {"bf16": {32: 16, 64: 16, 96: 16, 128: 12, 160: 12, 192: 8, 224: 8, 256: 8},
         "f16": {32: 16, 64: 16, 96: 12, 128: 12, 160: 8, 192: 8, 224: 8, 256: 8},
         "f32": {32: 16, 64: 16, 96: 12, 128: 8, 160: 8, 192: 8}}


@pytest.mark.parametrize("dtype,d", [(t, d) for t in WAVES for d in WAVES[t]])
def test_work_groups_that_fill_a_cu(dtype, d):
    """More than 128 sequences of few rows: their waves' states are joined in LDS, in halves.  One
    sequence is long enough for every wave, others leave waves without a tile, one has none."""
    need_gpu()
    lens = (1000, 0, 1, 300, 33) + tuple(5 + i % 60 for i in range(135))
    case = Case(d, lens, 1, d, 64)
    case.fill_tokens()
    q = normal(case.g, (len(lens), 3, 2, d), dtype)
    say("attend wide", dtype, d)
    x = launch(case, q)
    assert (x.many, x.rows, x.waves, x.splits) == (0, 16, WAVES[dtype][d], 1)
    run(case, q, dtype=dtype)
    run(case, q[:, :1].contiguous(), dtype=dtype, causal=False)


def two_groups(case, q):
    x = launch(case, q, "two")
    assert (x.many, x.rows) == (0, 32) and x.splits > 1


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_two_groups_query_that_is_not_finite(dtype, d, bad):
    """Its own row is NaN, the other rows keep their bits."""
    need_gpu()
    case = Case(37, (90, 200), 2, d, 32)
    case.fill_tokens()
    q = normal(case.g, (2, 20, 6, d), dtype)
    two_groups(case, q)
    O, LSE = run(case, q, kind="two", dtype=dtype)
    q2 = q.clone()
    q2[1, 7, 4, 50] = bad
    O2, LSE2 = run(case, q2, check=False, kind="two")
    assert O2[1, 7, 4].isnan().all() and LSE2[1, 4, 7].isnan()
    O2[1, 7, 4], LSE2[1, 4, 7] = O[1, 7, 4], LSE[1, 4, 7]
    assert torch.equal(O2, O) and torch.equal(LSE2, LSE)


def test_two_groups_result_over_the_queries():
    need_gpu()
    case = Case(67, (300, 65), 2, 64, 64)
    case.fill_tokens()
    q = normal(case.g, (2, 10, 8, 64), "bf16")
    two_groups(case, q)
    O, _ = run(case, q, kind="two")
    x = q.cuda()
    cq.cqsa_cache_attend(case.cache(), bounded(case, "two"), x, x)
    assert torch.equal(x, O)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_two_groups_not_a_number_reaches_only_rows_that_see_it(dtype):
    need_gpu()
    n, G, d = 33, 3, 64
    for what, at in (("k", 175), ("v", 175), ("v", 199), ("k", 199), ("v", 40)):
        case = Case(31, (200,), 4, d, 64)
        rows = case.fill_tokens()
        q = normal(case.g, (1, n, 4 * G, d), dtype)
        if what == "k" and at == 175:
            two_groups(case, q)
        O, LSE = run(case, q, kind="two", dtype=dtype)
        k, v = (x.copy() for x in rows[0])
        (k if what == "k" else v)[at, :, 35] = np.nan if at == 175 else np.inf
        p, t = case.slots(0, 0, 200)
        o4.write(case.data, 64, k, v, p, t)
        O2, LSE2 = run(case, q, check=False, kind="two")
        for i in range(n):
            if at > 200 - n + i:
                assert torch.equal(O2[0, i], O[0, i]) and torch.equal(LSE2[0, :, i], LSE[0, :, i])
            elif what == "k":
                assert O2[0, i].isnan().all() and LSE2[0, :, i].isnan().all()
            else:
                assert O2[0, i, :, 32:].isnan().all()
                assert torch.equal(O2[0, i, :, :32], O[0, i, :, :32])
                assert torch.equal(LSE2[0, :, i], LSE[0, :, i])


def test_two_groups_captured():
    """Replays follow the lengths and rows on the device, with a workspace of any contents."""
    need_gpu()
    H, G, d, n, lens = 2, 4, 64, 10, (700, 64)
    case = Case(53, lens, H, d, 64)
    case.fill_tokens()
    cache, batch = case.cache(), bounded(case, "two")
    q = normal(case.g, (2, n, H * G, d), "bf16").cuda()
    two_groups(case, q)
    O, LSE = torch.empty_like(q), torch.empty((2, H * G, n), device="cuda")
    space = cq.cqsa_cache_attend_workspace(cache, batch, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cq.cqsa_cache_attend(cache, batch, q, O, LSE, workspace=space)
    for cut in (0, 1, 29):
        now = [max(x - cut, 0) for x in lens]
        batch.lengths.copy_(torch.tensor(now, dtype=torch.int32))
        fresh = normal(case.g, (2, n, H * G, d), "bf16")
        q.copy_(fresh)
        space.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone(), LSE.clone()
        for b, x in enumerate(now):
            ref = reference(case, synth.as_f64(fresh)[b], b, x, True)
            held("bf16", O[b].cpu().double().numpy(), LSE[b].t().cpu().double().numpy(), ref, max(x, 1))
        O.zero_()
        cq.cqsa_cache_attend(cache, batch, q, O, LSE, workspace=space)
        torch.cuda.synchronize()
        assert torch.equal(O, got[0]) and torch.equal(LSE, got[1])


@pytest.mark.parametrize("dtype,B,G,chunk", [("f32", 1024, 4, 1100), ("bf16", 2048, 8, 300)])
def test_more_work_groups_than_one_dimension_takes(dtype, B, G, chunk):
    """A chunk beside single tokens of many sequences, max_q far above both: 2^24 work groups of the
    kernel for few rows, 2^22 of that for many.  Rows behind the last sequence stay as they were."""
    need_gpu()
    H, d, T = 8, 32, 8192
    lens = (chunk + 50,) + tuple(b % 7 for b in range(1, B))
    case = Case(B, lens, H, d, 32)
    case.fill_tokens()
    start = np.concatenate([[0], chunk + np.arange(B)]).astype(np.int32)
    q = normal(case.g, (1, T, H * G, d), dtype)
    batch = case.batch(q_start=torch.from_numpy(start).cuda(), max_q=T)
    say("attend wide grid", dtype, B, G, chunk)
    x = cq.cqsa_cache_attend_launch(case.cache(), batch, q.cuda())
    assert x.many == (dtype == "bf16") and B * H * (T * G // x.rows) * x.splits > 1 << 21
    O, LSE = torch.full_like(q, 9.0, device="cuda"), torch.full((1, H * G, T), 9.0, device="cuda")
    cq.cqsa_cache_attend(case.cache(), batch, q.cuda(), O, LSE)
    o, l = O[0].cpu().double().numpy(), LSE[0].t().cpu().double().numpy()
    for b in [0] + list(range(1, B, 97)) + [B - 1]:
        r = slice(start[b], start[b + 1])
        held(dtype, o[r], l[r], reference(case, synth.as_f64(q[:, r].contiguous())[0], b, lens[b], True), max(lens[b], 1))
    assert (o[start[-1]:] == 9).all() and (l[start[-1]:] == 9).all()


@pytest.mark.parametrize("n,G,B,H,longest,splits", [(40, 3, 64, 4, 400, 1), (64, 4, 33, 4, 500, 1), (140, 4, 13, 4, 1000, 2)])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_of_fp16_at_the_widest_head(n, G, B, H, longest, splits, causal):
    """fp16 at d = 256 in the kernel for many rows: ends inside work groups, sequences of fewer tokens
    than rows, of one and of none, and parts."""
    need_gpu()
    d = 256
    lens = (longest, 0, 1, 70) + tuple(3 + 11 * (i % 4) for i in range(B - 4))
    case = Case(n, lens, H, d, 32)
    case.fill_tokens()
    q = normal(case.g, (B, n, H * G, d), "f16")
    most = max(longest, 1024 if splits > 1 else 0)
    columns = np.full((B, -(-most // 32)), -1, np.int32)
    columns[:, :case.table.shape[1]] = case.table[:, :columns.shape[1]]
    case.table = columns
    say("attend many f16 256", n, G, B, H, longest, causal)
    x = launch(case, q)
    assert (x.many, x.rows, x.splits) == (1, 128, splits)
    run(case, q, dtype="f16", causal=causal)


@pytest.mark.parametrize("rows,tokens,many", [(128, 512, 1), (128, 513, 0), (112, 300, 1), (111, 300, 0), (80, 200, 0),
                                              (512, 1024, 1), (512, 1025, 0), (520, 1000, 0), (600, 1000, 1)])
def test_when_fp16_at_the_widest_head_takes_the_kernel_for_many(rows, tokens, many):
    need_gpu()
    table = torch.zeros((64, 40), dtype=torch.int32, device="cuda")
    batch = cq.CacheBatch(table, table[:, 0].contiguous(), max_len=tokens)
    q = torch.empty((64, rows, 8, 256), dtype=torch.float16, device="cuda")
    assert cq.cqsa_cache_attend_launch(cq.Cache4(1, 8, 256, page_size=32), batch, q).many == many
