"""Attention over the 4-bit cache on the GPU, against oracle.cache4 in float64.

Bounds, from the arithmetic.  With t = the largest sum of |q k| scale of a key
that the row sees: a score is off by at most e = t (2^-20 + d 2^-23): the scale,
its products and the change to powers of two round by under 2^-20 of it, the
products of its d terms are exact or rounded by half a step, and add up in fp32
with an error of at most half a step each.  LSE is then off by e, and by 2^-22
(|LSE| + 8) for the logarithm, the sum and the shift.  The weights are off by
2 e and their rounding u relative to themselves (u = 2^-8 for bf16, whose
weights enter the product rounded to bf16; 2^-16 for fp16, which takes two such
parts; 2^-22 for fp32, which takes three), so O by (2 e + u + n 2^-23) times
the weighted sum of |v|, n the tokens, and half a step of its type.  A weight
below 2^-126 of the largest is no normal fp32 number and may count as 0; the
values here are under 2^6, so n of them are n 2^-120 at most.
"""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import cache4 as o4
from oracle import rotary as orot
from paper_2604_20819_amd import synth
from tests.gpu_util import need_gpu, say
from tests.op_util import DT, HALF_STEP, Case, normal, starts

pytestmark = pytest.mark.gpu
WEIGHT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -16, "f32": 2.0 ** -22}


def held(dtype, O, LSE, ref, tokens):
    """O [n, Hq, d] and LSE [n, Hq] (numpy float64) of one sequence against the oracle's."""
    wo, wl, absv, big = ref
    d = O.shape[-1]
    e = big * (2.0 ** -20 + d * 2.0 ** -23)
    empty = np.isneginf(wl)
    assert np.array_equal(np.isneginf(LSE), empty)
    assert (O[empty] == 0).all()
    off = np.abs(np.where(empty, 0, LSE) - np.where(empty, 0, wl))
    assert (off <= e + 2.0 ** -22 * (np.abs(np.where(empty, 0, wl)) + 8)).all(), off.max()
    bound = (2 * e[..., None] + WEIGHT[dtype] + tokens * 2.0 ** -23) * absv + tokens * 2.0 ** -120
    bound = bound + HALF_STEP[dtype] * (np.abs(wo) + bound)
    if dtype == "f16":
        bound += 2.0 ** -25
    off = np.abs(O - wo)
    assert (off <= bound).all(), (off - bound).max()


# The launch goes by the lengths' bound, so a bound far above the lengths takes short
# sequences through the kernels and splits that long ones get: one group of 16 rows a
# wave, two, the kernel for many rows (more than 64).
BOUNDS = {"few": 0, "two": 1 << 17, "many": 1 << 22}


def run(case, q, lens=None, causal=True, scale=0.0, cache=None, dtype="bf16", check=True, kind="few", **kw):
    """The call on uniform rows q [B, n, Hq, d]; checked against the oracle."""
    B, n, Hq, d = q.shape
    cache = cache or case.cache()
    batch = bounded(case, kind, lens=lens, **kw)
    O = torch.full_like(q, 9.0, device="cuda")
    LSE = torch.full((B, Hq, n), 9.0, device="cuda")
    cq.cqsa_cache_attend(cache, batch, q.cuda(), O, LSE, causal=causal, scale=scale)
    torch.cuda.synchronize()
    if check:
        for b in range(B):
            length = (lens or case.lens)[b]
            ref = reference(case, synth.as_f64(q)[b], b, length, causal, scale)
            held(dtype, O[b].cpu().double().numpy(), LSE[b].t().cpu().double().numpy(), ref, max(length, 1))
    return O, LSE


def bounded(case, kind, lens=None, **kw):
    """The batch with a wide table where the bound needs one."""
    if not BOUNDS[kind]:
        return case.batch(lens=lens, **kw)
    wide = np.full((case.table.shape[0], BOUNDS[kind] // case.page), -1, np.int32)
    wide[:, :case.table.shape[1]] = case.table
    return cq.CacheBatch(torch.from_numpy(wide).cuda(),
                         torch.tensor(case.lens if lens is None else lens, dtype=torch.int32, device="cuda"),
                         **{"max_len": BOUNDS[kind], **kw})


def reference(case, q, b, length, causal, scale=0.0):
    p, t = case.slots(b, 0, length)
    k, v = o4.read(case.data, case.page, case.H, case.d, p, t)
    there = (p >= 0) & (p < case.n_pages)
    return o4.attend(q, k, v, there, length, causal, scale if scale > 0 else 1 / np.sqrt(case.d))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_one_token(dtype, d):
    """The next token of sequences of every short length, one query head a key head."""
    need_gpu()
    lens = (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 0, 129)
    case = Case(d, lens, 2, d, 64)
    case.fill_tokens()
    say("attend one", dtype, d)
    run(case, normal(case.g, (len(lens), 1, 2, d), dtype), dtype=dtype)


@pytest.mark.parametrize("G,n,page", [(1, 2, 32), (3, 5, 64), (8, 1, 128), (16, 1, 32), (17, 1, 64),
                                      (5, 7, 256), (4, 16, 64), (8, 33, 32), (2, 130, 128)])
@pytest.mark.parametrize("causal", [True, False])
def test_groups_and_rows(G, n, page, causal):
    """Grouped heads and several rows a sequence; short sequences have rows before position 0."""
    need_gpu()
    lens = (n - 1, 97, 300, 1)
    d, H = 64, 2
    case = Case(G * n, lens, H, d, page)
    case.fill_tokens()
    say("attend rows", G, n, page, causal)
    run(case, normal(case.g, (len(lens), n, G * H, d), "bf16"), causal=causal)


@pytest.mark.parametrize("dtype,d,G,n", [("f16", 128, 4, 9), ("f32", 96, 3, 40), ("f32", 256, 2, 65),
                                         ("bf16", 256, 8, 20), ("f16", 32, 1, 200), ("bf16", 160, 2, 150),
                                         ("f32", 224, 1, 17), ("bf16", 128, 16, 70)])
def test_types_and_rows(dtype, d, G, n):
    need_gpu()
    lens = (200, 333)
    case = Case(d + n, lens, 1, d, 64)
    case.fill_tokens()
    say("attend types", dtype, d, G, n)
    run(case, normal(case.g, (2, n, G, d), dtype), dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_many_rows(dtype, d):
    """The kernel for many rows: rows that end inside a wave and a work group, a sequence of fewer
    tokens than rows, one of none."""
    need_gpu()
    lens, n, G = (307, 70, 0), 97, 3
    case = Case(d + 7, lens, 1, d, 32)
    case.fill_tokens()
    say("attend many", dtype, d)
    q = normal(case.g, (3, n, G, d), dtype)
    run(case, q, dtype=dtype, kind="many")
    run(case, q[:, :25].contiguous(), dtype=dtype, kind="many", causal=False)


@pytest.mark.parametrize("dtype,d,kind,n", [("bf16", 128, "two", 5), ("f16", 96, "two", 9), ("bf16", 64, "two", 15),
                                            ("f16", 32, "two", 5), ("bf16", 128, "many", 40), ("f16", 64, "many", 70)])
def test_split_rows(dtype, d, kind, n):
    """Two groups of 16 rows a wave, and many rows, over contexts that are split."""
    need_gpu()
    lens, G = (3001, 64, 1499), 4
    case = Case(d + n, lens, 2, d, 64)
    case.fill_tokens()
    say("attend split", dtype, d, kind, n)
    run(case, normal(case.g, (3, n, 2 * G, d), dtype), dtype=dtype, kind=kind)


def test_kinds_take_the_launches_that_the_tests_mean():
    """By the workspace: a split call has one."""
    need_gpu()
    case = Case(3, (300, 70), 1, 64, 32)
    case.fill_tokens()
    for kind in BOUNDS:
        q = torch.zeros((2, 70, 2, 64), dtype=torch.bfloat16, device="cuda")
        space = cq.cqsa_cache_attend_workspace(case.cache(), bounded(case, kind), q)
        assert (space is None) == (kind == "few")


@pytest.mark.parametrize("n,kind", [(1, "few"), (3, "two"), (30, "many")])
def test_result_over_the_queries(n, kind):
    """O may be Q."""
    need_gpu()
    case = Case(67, (300, 65), 2, 64, 64)
    case.fill_tokens()
    q = normal(case.g, (2, n, 8, 64), "bf16")
    O, _ = run(case, q, kind=kind)
    x = q.cuda()
    cq.cqsa_cache_attend(case.cache(), bounded(case, kind), x, x)
    assert torch.equal(x, O)


@pytest.mark.parametrize("lens,n,G,B_pad", [((20011,), 1, 4, 0), ((9000, 17, 4097), 3, 2, 0),
                                            ((6000,), 40, 1, 30), ((2500, 5000), 1, 16, 60),
                                            ((2000, 40), 1, 16, 150), ((900, 333), 2, 3, 0)])
def test_long_contexts(lens, n, G, B_pad):
    """Contexts that are split over work groups, alone and beside many short sequences."""
    need_gpu()
    lens = lens + (3,) * B_pad
    d, H = 64, 1
    case = Case(len(lens), lens, H, d, 128)
    case.fill_tokens()
    say("attend long", lens[:3], n, G, B_pad)
    run(case, normal(case.g, (len(lens), n, G, d), "bf16"))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 192), ("bf16", 256)])
def test_many_rows_of_a_long_context(dtype, d):
    """One key head's long context spread over the whole GPU, beside one that leaves most parts empty."""
    need_gpu()
    lens, n, G = (40001, 33), 25, 4
    case = Case(71 + d, lens, 1, d, 256)
    case.fill_tokens()
    say("attend many long", dtype, d)
    run(case, normal(case.g, (2, n, G, d), dtype), dtype=dtype, kind="many")


@pytest.mark.parametrize("kind,G,dtype", [("few", 3, "bf16"), ("few", 3, "f32"), ("two", 1, "f16"), ("many", 3, "bf16")])
def test_packed_rows(kind, G, dtype):
    """Ragged rows; rows of no sequence stay as they were, LSE's too."""
    need_gpu()
    lens, new, first = (70, 40, 333, 3, 128), (65, 0, 1, 9, 128), 3
    H, d = 2, 96
    if kind == "two":  # as many rows as that takes
        lens, new = (70, 40, 333, 3, 60), (55, 0, 1, 9, 60)
    case = Case(17, lens, H, d, 32)
    case.fill_tokens()
    T = first + sum(new) + 4
    q = normal(case.g, (1, T, H * G, d), dtype)
    batch = bounded(case, kind, q_start=starts(new, first), max_q=max(new))
    O = torch.full_like(q, 9.0, device="cuda")
    LSE = torch.full((1, H * G, T), 9.0, device="cuda")
    cq.cqsa_cache_attend(case.cache(), batch, q.cuda(), O, LSE)
    off = first + np.concatenate([[0], np.cumsum(new)])
    o, l = O[0].cpu().double().numpy(), LSE[0].t().cpu().double().numpy()
    for b, n in enumerate(lens):
        r = slice(off[b], off[b + 1])
        held(dtype, o[r], l[r], reference(case, synth.as_f64(q)[0, r], b, n, True), n)
    for x in (o, l):
        assert (x[:first] == 9).all() and (x[off[-1]:] == 9).all()


@pytest.mark.parametrize("kind,rows", [("few", (1, 50)), ("two", (17,)), ("many", (33, 150))])
def test_given_up_pages_and_bad_entries(kind, rows):
    """Entries outside the pool hold no tokens; a sequence of only such ones is empty."""
    need_gpu()
    lens, d = (200, 130, 64, 70), 64
    case = Case(23, lens, 1, d, 32)
    case.fill_tokens()
    case.table[0, 0:2] = -1
    case.table[0, 4] = case.n_pages + 7
    case.table[1, 4] = -2 ** 31
    case.table[2, :] = 2 ** 31 - 1
    for n in rows:
        run(case, normal(case.g, (4, n, 2, d), "bf16"), kind=kind)


@pytest.mark.parametrize("kind", ["few", "two", "many"])
def test_starts_that_fall(kind):
    """Rows that two sequences share get results of any; the others are right, and none of no
    sequence is written."""
    need_gpu()
    lens, G, d = (60, 70, 80), 4, 64
    case = Case(83, lens, 1, d, 32)
    case.fill_tokens()
    q = normal(case.g, (1, 60, G, d), "bf16")
    batch = bounded(case, kind, q_start=torch.tensor([3, 30, 20, 55], dtype=torch.int32).cuda(), max_q=40)
    O = torch.full_like(q, 9.0, device="cuda")
    LSE = torch.full((1, G, 60), 9.0, device="cuda")
    cq.cqsa_cache_attend(case.cache(), batch, q.cuda(), O, LSE)
    o, l = O[0].cpu().double().numpy(), LSE[0].t().cpu().double().numpy()
    for b, lo, hi, first, last in ((0, 3, 30, 3, 20), (2, 20, 55, 30, 55)):
        ref = reference(case, synth.as_f64(q)[0, lo:hi], b, lens[b], True)
        held("bf16", o[first:last], l[first:last], [x[first - lo:last - lo] for x in ref], lens[b])
    for x in (o, l):
        assert (x[:3] == 9).all() and (x[55:] == 9).all()


def test_no_pages_and_no_tokens():
    """A pool of no pages, and a table of no columns: nothing is seen."""
    need_gpu()
    empty = cq.Cache4(0, 2, 64, page_size=32)
    lengths = torch.tensor([5, 0], dtype=torch.int32, device="cuda")
    q = torch.ones((2, 3, 4, 64), dtype=torch.float16, device="cuda")
    k, v = torch.full((2, 2, 3, 2, 64), 9.0, dtype=torch.float16, device="cuda")
    for columns in (0, 1):
        batch = cq.CacheBatch(torch.zeros((2, columns), dtype=torch.int32, device="cuda"), lengths)
        O, LSE = torch.full_like(q, 9.0), torch.full((2, 4, 3), 9.0, device="cuda")
        cq.cqsa_cache_write(empty, batch, k, v)
        cq.cqsa_cache_attend(empty, batch, q, O, LSE)
        assert (O == 0).all() and LSE.isneginf().all()
        ko, vo = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
        cq.cqsa_cache_read(empty, batch, ko, vo)
        assert (ko == 0).all() and (vo == 0).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f16", 224), ("bf16", 256), ("f16", 256)])
def test_many_sequences_of_many_rows(dtype, d):
    """Whole short prompts, whose work groups fill the GPU: the kernel for many rows without splits."""
    need_gpu()
    lens, n, H = tuple(80 - 7 * (i % 9) for i in range(64)), 80, 4
    case = Case(89, lens, H, d, 32)
    case.fill_tokens()
    run(case, normal(case.g, (64, n, H, d), dtype), dtype=dtype)


def test_lengths_out_of_range():
    need_gpu()
    case = Case(29, (96, 96, 96), 1, 64, 32)
    case.fill_tokens()
    q = normal(case.g, (3, 2, 1, 64), "bf16")
    O, LSE = run(case, q, lens=[2 ** 31 - 1, -4, 50], check=False, max_len=80)
    for b, n in enumerate((80, 0, 50)):
        ref = reference(case, synth.as_f64(q)[b], b, n, True)
        held("bf16", O[b].cpu().double().numpy(), LSE[b].t().cpu().double().numpy(), ref, max(n, 1))


@pytest.mark.parametrize("n,G,kind", [(1, 1, "few"), (6, 1, "few"), (70, 2, "few"), (20, 1, "two"),
                                      (70, 2, "two"), (70, 2, "many"), (290, 1, "many"), (199, 1, "many")])
def test_not_a_number_reaches_only_rows_that_see_it(n, G, kind):
    """A NaN or an infinity in a key makes the rows that see it NaN; in a value, their 32 channels;
    other rows keep their bits."""
    need_gpu()
    d, H = 64, 1
    for what, at in (("k", 150), ("v", 150), ("v", 199), ("k", 199), ("v", 40)):
        case = Case(31, (200,), H, d, 64)
        rows = case.fill_tokens()
        q = normal(case.g, (1, n, G, d), "bf16")
        O, LSE = run(case, q, kind=kind)
        k, v = (x.copy() for x in rows[0])
        (k if what == "k" else v)[at, 0, 35] = np.nan if at == 150 else np.inf
        p, t = case.slots(0, 0, 200)
        o4.write(case.data, 64, k, v, p, t)
        O2, LSE2 = run(case, q, check=False, kind=kind)
        for i in range(n):
            sees = at <= 200 - n + i
            same = torch.equal(O2[0, i], O[0, i]) and torch.equal(LSE2[0, :, i], LSE[0, :, i])
            assert same or sees, (what, at, i)
            if sees and what == "k":
                assert O2[0, i].isnan().all() and LSE2[0, :, i].isnan().all()
            elif sees:
                assert O2[0, i, :, 32:].isnan().all()
                assert torch.equal(O2[0, i, :, :32], O[0, i, :, :32])
                assert torch.equal(LSE2[0, :, i], LSE[0, :, i])


@pytest.mark.parametrize("kind", ["few", "two", "many"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_query_that_is_not_finite(bad, kind):
    """Its own row is NaN, the other rows keep their bits."""
    need_gpu()
    case = Case(37, (90,), 1, 64, 32)
    case.fill_tokens()
    q = normal(case.g, (1, 23, 3, 64), "bf16")
    O, LSE = run(case, q, kind=kind)
    q2 = q.clone()
    q2[0, 7, 1, 50] = bad
    O2, LSE2 = run(case, q2, check=False, kind=kind)
    assert O2[0, 7, 1].isnan().all() and LSE2[0, 1, 7].isnan()
    O2[0, 7, 1], LSE2[0, 1, 7] = O[0, 7, 1], LSE[0, 1, 7]
    assert torch.equal(O2, O) and torch.equal(LSE2, LSE)


@pytest.mark.parametrize("gain,scale", [(1e-20, 0.0), (1e4, 0.0), (1.0, 7.5), (1.0, 1e-6)])
def test_sizes_of_scores(gain, scale):
    """Weights all alike, or one of them everything: scores from nothing to thousands."""
    need_gpu()
    case = Case(41, (300, 77), 1, 64, 32)
    case.fill_tokens(gain)
    run(case, normal(case.g, (2, 5, 2, 64), "f32"), dtype="f32", scale=scale)


def test_query_elements_of_many_sizes():
    """A block's elements from its largest down to 2^-40 of it."""
    need_gpu()
    case = Case(43, (200,), 1, 128, 32)
    case.fill_tokens()
    for dtype in ("bf16", "f32"):
        q = torch.randn(1, 3, 2, 128, generator=torch.Generator().manual_seed(1))
        q = (q * 2.0 ** -torch.arange(128).remainder(41)).to(DT[dtype])
        run(case, q, dtype=dtype)


def test_strided_and_without_lse():
    need_gpu()
    B, n, Hq, d = 2, 9, 4, 128
    case = Case(47, (50, 81), 2, d, 64)
    case.fill_tokens()
    q = normal(case.g, (B, n, Hq, d), "f16")
    O, _ = run(case, q, dtype="f16")
    wide = torch.full((B, n, Hq + 3, d), 9.0, dtype=torch.float16, device="cuda")
    wide[:, :, 1:1 + Hq] = q.cuda()
    out = torch.full((B, Hq, n, 2 * d), 9.0, dtype=torch.float16, device="cuda")
    view = out[..., d:].transpose(1, 2)
    cq.cqsa_cache_attend(case.cache(), case.batch(), wide[:, :, 1:1 + Hq], view)
    assert torch.equal(view, O) and (out[..., :d] == 9).all()


@pytest.mark.parametrize("n,lens,kind", [(1, (5000, 30), "few"), (64, (700, 64), "few"), (8, (700, 64), "two"),
                                         (40, (1700, 64), "many")])
def test_captured_on_streams_and_repeated(n, lens, kind):
    """Replays follow the lengths, tables and rows on the device; the same call gives the same
    bits on any stream, with a workspace of any contents."""
    need_gpu()
    H, G, d = 1, 4, 64
    case = Case(53, lens, H, d, 64)
    case.fill_tokens()
    cache = case.cache()
    batch = bounded(case, kind, max_len=BOUNDS[kind] or case.table.shape[1] * 64)
    q = normal(case.g, (2, n, G, d), "bf16").cuda()
    O, LSE = torch.empty_like(q), torch.empty((2, G, n), device="cuda")
    space = cq.cqsa_cache_attend_workspace(cache, batch, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cq.cqsa_cache_attend(cache, batch, q, O, LSE, workspace=space)
    for cut in (0, 1, 29):
        now = [max(x - cut, 0) for x in lens]
        batch.lengths.copy_(torch.tensor(now, dtype=torch.int32))
        fresh = normal(case.g, (2, n, G, d), "bf16")
        q.copy_(fresh)
        if space is not None:
            space.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        got = O.clone(), LSE.clone()
        for b, x in enumerate(now):
            ref = reference(case, synth.as_f64(fresh)[b], b, x, True)
            held("bf16", O[b].cpu().double().numpy(), LSE[b].t().cpu().double().numpy(), ref, max(x, 1))
        for stream in (None, s.cuda_stream):
            O.zero_()
            torch.cuda.synchronize()
            cq.cqsa_cache_attend(cache, batch, q, O, LSE, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(O, got[0]) and torch.equal(LSE, got[1])


@pytest.mark.parametrize("n,kind", [(1, "few"), (30, "many")])
def test_two_calls_at_once(n, kind):
    """Calls on two streams, and graphs captured without a workspace of the caller's, side by side."""
    need_gpu()
    G, d, jobs = 4, 64, []
    for seed in (97, 101):
        case = Case(seed, (6000, 900), 1, d, 64)
        case.fill_tokens()
        q = normal(case.g, (2, n, G, d), "bf16")
        want, _ = run(case, q, kind=kind)
        jobs.append((case.cache(), bounded(case, kind), q.cuda(), torch.empty_like(want), want))
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, (cache, batch, q, O, _) in zip(streams, jobs):
            cq.cqsa_cache_attend(cache, batch, q, O, stream=s.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(O, want) for _, _, _, O, want in jobs)
    graphs = []
    for s, (cache, batch, q, O, _) in zip(streams, jobs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=s):
            cq.cqsa_cache_attend(cache, batch, q, O)
        O.zero_()
    torch.cuda.synchronize()
    for _ in range(8):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(O, want) for _, _, _, O, want in jobs)


def test_pages_beyond_four_gigabytes():
    need_gpu()
    H, d, page = 8, 128, 256
    per = cq.cqsa_cache_page_bytes(page, H, d)
    n_pages = (9 << 29) // per
    cache = cq.Cache4(n_pages, H, d, page_size=page, data=torch.zeros((n_pages, per), dtype=torch.uint8, device="cuda"))
    case = Case(59, (300,), H, d, page, spare=0, extra_columns=0)
    rows = case.fill_tokens()
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    for j in range(2):
        cache.data[n_pages - 1 - j] = torch.from_numpy(case.data[case.table[0, j]]).cuda()
    batch = cq.CacheBatch(table, torch.tensor([300], dtype=torch.int32, device="cuda"))
    for n in (1, 33):
        q = normal(case.g, (1, n, 16, d), "bf16")
        O, LSE = torch.empty_like(q, device="cuda"), torch.empty((1, 16, n), device="cuda")
        cq.cqsa_cache_attend(cache, batch, q.cuda(), O, LSE)
        ref = reference(case, synth.as_f64(q)[0], 0, 300, True)
        held("bf16", O[0].cpu().double().numpy(), LSE[0].t().cpu().double().numpy(), ref, 300)
    assert len(rows) == 1


def test_rotary_write_attend_together():
    """A prompt and five steps as a program serves them: rotary positions of three axes, the new
    keys and values into the cache, attention over it; and the cache read back for cqsa_forward."""
    need_gpu()
    B, Hq, H, d, page, prompt, steps = 2, 4, 2, 128, 32, 45, 5
    sections = (16, 24, 24)
    g = np.random.Generator(np.random.PCG64(61))
    case = Case(61, (prompt + steps,) * B, H, d, page)
    cache, plan = case.cache(), cq.cqsa_rotary_plan(d, sections)
    total = prompt + steps
    qkv = torch.from_numpy(g.standard_normal((B, total, Hq + 2 * H, d), dtype=np.float32)).bfloat16()
    pos = torch.from_numpy(g.integers(0, 200000, (3, B, total)).astype(np.int32))
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(case.table).cuda()
    O = torch.empty((B, total, Hq, d), dtype=torch.bfloat16, device="cuda")
    turned = qkv.clone()
    for lo, hi in [(0, prompt)] + [(t, t + 1) for t in range(prompt, total)]:
        w = qkv[:, lo:hi].cuda()
        q, k, v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
        cq.cqsa_rotary(plan, pos[:, :, lo:hi].contiguous().cuda(), [q, k])
        lengths.fill_(hi)
        batch = cq.CacheBatch(table, lengths)
        cq.cqsa_cache_write(cache, batch, k, v)
        cq.cqsa_cache_attend(cache, batch, q, O[:, lo:hi])
        turned[:, lo:hi] = w.cpu()
    want, size = orot.rotate(synth.as_f64(qkv[:, :, :Hq + H].contiguous()), pos.numpy(), sections)
    bound = size * 2.0 ** -21 + HALF_STEP["bf16"] * (np.abs(want) + size * 2.0 ** -21)
    assert (np.abs(synth.as_f64(turned[:, :, :Hq + H].contiguous()) - want) <= bound).all()
    for b in range(B):
        t = synth.as_f64(turned[b])
        p, at = case.slots(b, 0, total)
        o4.write(case.data, page, t[:, Hq:Hq + H], t[:, Hq + H:], p, at)
        ref = reference(case, t[:, :Hq], b, total, True)
        held("bf16", O[b].cpu().double().numpy(), ref[1], ref, total)
    ko, vo = (torch.empty((B, total, H, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cq.cqsa_cache_read(cache, cq.CacheBatch(table, lengths), ko, vo)
    # the library's attention over what the cache holds: the same function, with its own roundings
    q = turned[:, :, :Hq].cuda()
    grown = [x.repeat_interleave(Hq // H, 2).contiguous() for x in (ko, vo)]
    Of, LSEf, _ = cq.forward(q.contiguous(), *grown, True)
    for b in range(B):
        ref = reference(case, synth.as_f64(turned[b, :, :Hq].contiguous()), b, total, True)
        held("bf16", Of[b].cpu().double().numpy(), LSEf[b].t().cpu().double().numpy(), ref, total)
