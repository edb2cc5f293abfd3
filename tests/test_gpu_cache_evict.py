"""cqsa_cache_evict against the oracle: every byte of the pool, every position and weight exactly."""
import math

import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import bounded as ob
from oracle import cache4 as o4
from tests.gpu_util import need_gpu, say
from tests.op_util import Case

pytestmark = pytest.mark.gpu


def random_bytes(case):
    """Bytes that no two tokens share (by chance): moving is all that is tested."""
    case.data = case.g.integers(0, 256, case.data.shape, dtype=np.uint8)


def bytes_of(data, page, d, H, p, t, h):
    return np.concatenate([data[p, i] for i in o4.places(page, d, h, int(t))])


def moved(case, W, budget, first, recent, target):
    """The pool, kept, lengths and weights after an eviction, by the definition; target: the tables written."""
    data = case.data.copy()
    B, H, d, page = len(case.lens), case.H, case.d, case.page
    kept = np.full((B, H, budget), -1, np.int32)
    lens = np.zeros(B, np.int32)
    Wn = W.copy()
    for b, n in enumerate(case.lens):
        p, t = case.slots(b, 0, n)
        there = (p >= 0) & (p < case.n_pages)
        for h in range(H):
            k = ob.keep(W[b, h], there, n, budget, first, recent)
            kept[b, h, :len(k)] = k
            lens[b] = len(k)
            for i, src in enumerate(k):
                Wn[b, h, i] = W[b, h, src]
                q = target[b, i // page]
                if 0 <= q < case.n_pages:
                    for x, y in zip(o4.places(page, d, h, i % page), o4.places(page, d, h, int(t[src]))):
                        data[q, x] = case.data[p[src], y]
    return data, kept, lens, Wn


def same(a, b):
    return np.array_equal(a.view(np.uint32), b.view(np.uint32))


def run(case, budget, first=0, recent=0, W=None, in_place=True, kept=True, alias=False, spare=5, max_len=0):
    B, H = len(case.lens), case.H
    T = case.table.shape[1] * case.page + spare
    if W is None:
        W = np.exp(2 * case.g.standard_normal((B, H, T))).astype(np.float32)
    cache, batch = case.cache(), case.batch(max_len=max_len)
    Wd = torch.from_numpy(W.copy()).cuda()
    k = torch.full((B, H, budget), 99, dtype=torch.int32, device="cuda") if kept else None
    new = batch.lengths if alias else torch.full((B,), -5, dtype=torch.int32, device="cuda")
    if in_place:
        cq.cqsa_cache_evict(cache, batch, Wd, new, budget, first, recent, kept=k)
        target, W_to = case.table, Wd
    else:
        target = case.target
        W_to = torch.full((B, H, T), 7.0, device="cuda")
        cq.cqsa_cache_evict(cache, batch, Wd, new, budget, first, recent, kept=k,
                            to=torch.from_numpy(target).cuda(), W_to=W_to)
    torch.cuda.synchronize()
    data, kk, lens, Wn = moved(case, W, budget, first, recent, target)
    assert np.array_equal(new.cpu().numpy(), lens)
    if kept:
        assert np.array_equal(k.cpu().numpy(), kk)
    got = W_to.cpu().numpy()
    if in_place:
        assert same(got, Wn)
    else:
        assert same(Wd.cpu().numpy(), W)
        for b, n in enumerate(lens):
            assert same(got[b, :, :n].copy(), Wn[b, :, :n].copy()) and (got[b, :, n:] == 7).all()
    assert np.array_equal(cache.data.cpu().numpy(), data)


def case_of(seed, lens, H, d, page, budget=None):
    """A pool with pages for the target too."""
    need = sum(-(-min(n, budget) // page) for n in lens) if budget else 0
    case = Case(seed, lens, H, d, page, spare=2 + need)
    random_bytes(case)
    if budget:
        free = np.setdiff1d(np.arange(case.n_pages), case.table[case.table >= 0])
        free = case.g.permutation(free)
        case.target = np.full((len(lens), -(-min(budget, case.table.shape[1] * page) // page) + 1), -1, np.int32)
        at = 0
        for b, n in enumerate(lens):
            m = -(-min(n, budget) // page)
            case.target[b, :m] = free[at:at + m]
            at += m
    return case


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_head_dims(d, in_place):
    need_gpu()
    say("evict", d, in_place)
    run(case_of(d, [150, 40, 41, 1, 0], 2, d, 32, 40), 40, 2, 7, in_place=in_place)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("page", [32, 64, 128, 256])
@pytest.mark.parametrize("budget,first,recent", [(1, 0, 0), (1, 1, 0), (33, 0, 33), (100, 100, 0), (64, 3, 20), (500, 1, 1)])
def test_budgets(page, budget, first, recent, in_place):
    need_gpu()
    say("evict budgets", page, budget, first, recent, in_place)
    run(case_of(budget + page, [300, 99, 33], 3, 32, page, budget), budget, first, recent, in_place=in_place, kept=budget != 64)


def weird(case, T):
    """Ties, both zeros, negatives, infinities, NaN, subnormals, neighbours in the last bit."""
    x = np.array([0.0, -0.0, 1.0, 1.0, np.nextafter(np.float32(1), np.float32(2)), -1.0, np.inf, -np.inf, np.nan,
                  1e-42, -1e-42, 3.4e38, -3.4e38], np.float32)
    W = x[case.g.integers(0, len(x), (len(case.lens), case.H, T))]
    W[0, 0, 7:9] = np.array([0xffc00001, 0x7f800001], np.uint32).view(np.float32)
    return W


@pytest.mark.parametrize("budget", [1, 30, 77, 150, 199, 200])
def test_ties_and_numbers_that_are_none(budget):
    need_gpu()
    say("evict ties", budget)
    case = case_of(budget, [200, 180], 2, 32, 64)
    run(case, budget, 0, 1, W=weird(case, case.table.shape[1] * 64 + 5))
    case = case_of(budget, [200, 180], 2, 32, 64)
    run(case, budget, W=np.zeros((2, 2, case.table.shape[1] * 64 + 5), np.float32))


@pytest.mark.parametrize("in_place", [True, False])
def test_pages_that_hold_nothing(in_place):
    """Their tokens are never kept, first and recent ones neither; a target's dropped."""
    need_gpu()
    say("evict holes", in_place)
    case = case_of(3, [200, 100, 64, 70], 2, 64, 32, 60)
    case.table[0, 0] = -1
    case.table[0, 3] = 10 ** 6
    case.table[1, 3] = -9
    case.table[2, :2] = -1
    if not in_place:
        case.target[3, 1] = -1
        case.target[1, 0] = case.n_pages
    run(case, 60, 3, 10, in_place=in_place)


def test_lengths_in_place_and_bounds():
    need_gpu()
    say("evict alias")
    run(case_of(4, [130, 90], 2, 64, 32), 50, 2, 3, alias=True)
    case = case_of(5, [130, 90], 2, 64, 32)
    case.lens = [130, 90]
    run(case, 50, 2, 3, max_len=130, kept=False)
    # lengths outside their range are taken as the nearest ones
    case = case_of(6, [128, 0], 2, 64, 64)
    cache = case.cache()
    batch = cq.CacheBatch(torch.from_numpy(case.table).cuda(), torch.tensor([1 << 30, -3], dtype=torch.int32, device="cuda"),
                          max_len=128)
    W = torch.rand(2, 2, 128, device="cuda")
    want = W[0].topk(20, -1).indices.sort(-1).values.int()
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros(2, 2, 20, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, new, 20, kept=kept)
    assert new.tolist() == [20, 0] and torch.equal(kept[0], want) and (kept[1] == -1).all()


def test_nothing_to_evict():
    need_gpu()
    say("evict nothing")
    case = case_of(7, [90, 0], 1, 32, 32)
    run(case, 90)
    run(case, 200, 5, 5)


@pytest.mark.parametrize("n,budget,kind", [(70001, 20000, "random"), (70001, 69999, "random"), (40000, 1000, "zeros"),
                                           (66000, 33001, "two"), (16384, 4096, "random"), (16385, 5, "random")])
def test_long_sequences(n, budget, kind):
    """Against torch on the device: positions, weights and the bytes by the cache's own read."""
    need_gpu()
    say("evict long", n, budget, kind)
    H, d, page = 3, 32, 256
    m = -(-n // page)
    g = torch.Generator("cuda").manual_seed(n)
    data = torch.randint(0, 256, (m, cq.cqsa_cache_page_bytes(page, H, d)), generator=g, device="cuda", dtype=torch.uint8)
    tiles = data.view(m, -1, 34 * d)
    tiles[..., 32 * d:] = 120 + tiles[..., 32 * d:] % 8
    pages = torch.randperm(m, generator=g, device="cuda").int()[None].contiguous()
    lengths = torch.tensor([n], dtype=torch.int32, device="cuda")
    cache, batch = cq.Cache4(m, H, d, page_size=page, data=data), cq.CacheBatch(pages, lengths)
    W = torch.rand(1, H, m * page, generator=g, device="cuda")
    if kind == "zeros":
        W.zero_()
    if kind == "two":
        W = (W > 0.7).float()
    k, v = torch.empty(2, 1, n, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, batch, k, v)
    order = torch.sort(W[0, :, :n], dim=-1, descending=True, stable=True).indices[:, :budget].sort(-1).values
    old = W.clone()
    kept = torch.zeros(1, H, budget, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, lengths, budget, kept=kept)
    assert lengths.item() == budget and torch.equal(kept[0].long(), order)
    assert torch.equal(W[0, :, :budget], old[0].gather(1, order)) and torch.equal(W[..., budget:], old[..., budget:])
    k2, v2 = torch.empty(2, 1, budget, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, cq.CacheBatch(pages, lengths), k2, v2)
    for x, y in ((k, k2), (v, v2)):
        want = x[0].transpose(0, 1).gather(1, order[..., None].expand(-1, -1, d))
        assert torch.equal(y[0].transpose(0, 1), want)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n,budget", [(4000, 900), (5000, 4999), (16000, 3000), (20000, 150), (40000, 12000), (90000, 30011)])
def test_long_batches_with_holes_and_strange_weights(n, budget, in_place):
    """Every way of choosing: ties, NaN, infinities, pages that hold nothing, a sequence with none and one without tokens."""
    need_gpu()
    say("evict long batch", n, budget, in_place)
    H, d, page, first, recent = 2, 32, 128, 5, 100
    lens = [n, n // 3, 700, 0]
    need = [-(-x // page) for x in lens]
    g = torch.Generator("cuda").manual_seed(n)
    pool = sum(need) * 2 + 1
    order = torch.randperm(pool, generator=g, device="cuda").int()
    pages = torch.full((4, need[0] + 1), -1, dtype=torch.int32, device="cuda")
    to = pages.clone()
    for b, m in enumerate(need):
        pages[b, :m] = order[sum(need[:b]):sum(need[:b]) + m]
        to[b, :m] = order[sum(need) + sum(need[:b]):sum(need) + sum(need[:b]) + m]
    if not in_place:
        pages[0, [0, 3, need[0] - 1]] = -1
        pages[1, 2] = pool
        pages[2] = -5
    data = torch.randint(0, 256, (pool, cq.cqsa_cache_page_bytes(page, H, d)), generator=g, device="cuda", dtype=torch.uint8)
    data.view(pool, -1, 34 * d)[..., 32 * d:] = 124
    cache = cq.Cache4(pool, H, d, page_size=page, data=data)
    lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
    batch = cq.CacheBatch(pages, lengths, max_len=n)
    W = torch.randn(4, H, n + 3, generator=g, device="cuda")
    odd = torch.tensor([0.0, -0.0, math.nan, math.inf, -math.inf, 1e-42, 1.0, -1.0], device="cuda")
    pick = torch.randint(0, 40, W.shape, generator=g, device="cuda")
    W = torch.where(pick < 8, odd[pick.clamp(max=7)], W)
    k, v = torch.zeros(2, 4, n, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, batch, k, v)
    t = torch.arange(n, device="cuda")
    rank = torch.where(torch.isnan(W), -1e302, W.double().clamp(-1e301, 1e301))[..., :n]
    L = lengths[:, None]
    forced = (t < first) | (t >= L - recent)
    entry = pages[:, t // page]
    there = (t < L) & (entry >= 0) & (entry < pool)
    rank = rank.masked_fill(forced[:, None], 1e303).masked_fill(~there[:, None], -1e303)
    keep = there.sum(-1).clamp(max=budget)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    gone = (torch.arange(best.shape[-1], device="cuda") >= keep[:, None])[:, None]
    best = best.masked_fill(gone, n).sort(-1).values
    old, new = W.clone(), torch.zeros(4, dtype=torch.int32, device="cuda")
    kept = torch.full((4, H, budget), 9, dtype=torch.int32, device="cuda")
    W_to = None if in_place else torch.full((4, H, n), 7.0, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, new, budget, first, recent, to=None if in_place else to, W_to=W_to, kept=kept)
    assert torch.equal(new.long(), keep)
    assert torch.equal(kept.long(), torch.where(best < n, best, -1))
    after = cq.CacheBatch(pages if in_place else to, new, max_len=n)
    k2, v2 = torch.zeros(2, 4, budget, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, after, k2, v2)
    got = (W if in_place else W_to).view(torch.int32)
    for b in range(4):
        m = int(keep[b])
        for h in range(H):
            src = best[b, h, :m]
            assert torch.equal(got[b, h, :m], old[b, h].view(torch.int32)[src])
            row = n - lens[b] + src  # what was read ends with the sequence's last token
            assert torch.equal(k2[b, budget - m:, h], k[b, row, h]) and torch.equal(v2[b, budget - m:, h], v[b, row, h])


def test_more_sequences_and_heads_than_one_dimension_takes():
    need_gpu()
    say("evict many heads")
    B, H = 32768, 65
    cache = cq.Cache4(1, H, 32, page_size=64)
    g = torch.Generator("cuda").manual_seed(3)
    lengths = torch.randint(0, 33, (B,), generator=g, device="cuda", dtype=torch.int32)
    batch = cq.CacheBatch(torch.zeros(B, 1, dtype=torch.int32, device="cuda"), lengths, max_len=32)
    W = torch.rand(B, H, 32, generator=g, device="cuda")
    new = torch.zeros(B, dtype=torch.int32, device="cuda")
    kept = torch.zeros(B, H, 9, dtype=torch.int32, device="cuda")
    W_to = torch.full((B, H, 9), 7.0, device="cuda")
    nowhere = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, new, 9, to=nowhere, W_to=W_to, kept=kept)
    t = torch.arange(32, device="cuda")
    w = W.masked_fill(t >= lengths[:, None, None], -1)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :9]
    n = lengths.clamp(max=9)
    gone = (torch.arange(9, device="cuda") >= n[:, None])[:, None]
    want = order.masked_fill(gone, 99).sort(-1).values
    assert torch.equal(new, n) and torch.equal(kept.long(), torch.where(want == 99, -1, want))
    assert torch.equal(W_to, torch.where(gone, 7.0, W.gather(-1, want.clamp(max=31))))


def test_work_groups_of_several_chunks():
    """More long heads than get a work group for each of their chunks of 4096 tokens (2^22 in all): each goes through
    several.  The same weights for every sequence, of three lengths, as a call of three sequences keeps them."""
    need_gpu()
    say("evict many long heads")
    B, H, T, budget, first, recent = 65536, 2, 140003, 50, 2, 9
    cache = cq.Cache4(1, H, 32, page_size=256)
    pages = torch.zeros(B, -(-T // 256), dtype=torch.int32, device="cuda")
    pages[:, 7] = -1  # the first 256 tokens behind 1792 have no page
    assert B * H * -(-T // 4096) > 2 ** 22
    g = torch.Generator("cuda").manual_seed(5)
    W = torch.rand(1, H, T, generator=g, device="cuda")
    W = torch.where(W < 0.3, 0.25, W)
    W[:, 1] = (W[:, 1] * 8).floor()  # many equal ones
    lens = torch.tensor([T, 33000, 70001], dtype=torch.int32, device="cuda")
    lengths = lens[torch.arange(B, device="cuda") % 3].contiguous()
    nowhere = torch.full((B, 1), -1, dtype=torch.int32, device="cuda")

    def run(n, lengths):
        new = torch.zeros(n, dtype=torch.int32, device="cuda")
        kept = torch.full((n, H, budget), 7, dtype=torch.int32, device="cuda")
        W_to = torch.zeros(n, H, budget, device="cuda")
        cq.cqsa_cache_evict(cache, cq.CacheBatch(pages[:n], lengths, max_len=T), W.expand(n, -1, -1), new, budget, first, recent,
                            to=nowhere[:n], W_to=W_to, kept=kept)
        return new, kept, W_to

    few, many = run(3, lens), run(B, lengths)
    for b, n in enumerate(lens.tolist()):
        there = np.ones(n, bool)
        there[7 * 256:8 * 256] = False
        for h in range(H):
            assert few[1][b, h].tolist() == ob.keep(W[0, h].cpu().numpy(), there, n, budget, first, recent)
    for x, y in zip(few, many):
        assert torch.equal(y, x[torch.arange(B, device="cuda") % 3])


def test_weights_far_apart():
    """Weights and pages whose bytes lie past 2^31."""
    need_gpu()
    say("evict far")
    H, d, page = 2, 256, 256
    per = cq.cqsa_cache_page_bytes(page, H, d)
    m = 2 ** 31 // per + 40
    cache = cq.Cache4(m, H, d, page_size=page)
    pages = torch.tensor([[m - 1, m - 3], [m - 5, 1]], dtype=torch.int32, device="cuda")
    to = torch.tensor([[0], [m - 7]], dtype=torch.int32, device="cuda")
    g = torch.Generator("cuda").manual_seed(1)
    for i in pages.flatten().tolist():
        cache.data[i] = torch.randint(0, 256, (per,), generator=g, device="cuda", dtype=torch.uint8)
        cache.data[i].view(-1, 34 * d)[:, 32 * d:] = 120
    lengths = torch.tensor([500, 300], dtype=torch.int32, device="cuda")
    batch = cq.CacheBatch(pages, lengths)
    far = 2 ** 31 + 777
    store = torch.empty(far + 10 ** 5, device="cuda")
    W = store.as_strided((2, H, 512), (far, 600, 1))
    W.copy_(torch.rand(2, H, 512, generator=g, device="cuda"))
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    kept = torch.zeros(2, H, 200, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, new, 200, to=to, kept=kept)
    assert new.tolist() == [200, 200]
    k, v = torch.empty(2, 2, 500, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, batch, k, v)
    k2, v2 = torch.empty(2, 2, 200, H, d, device="cuda").unbind(0)
    cq.cqsa_cache_read(cache, cq.CacheBatch(to, new), k2, v2)
    for b, n in enumerate((500, 300)):
        for h in range(H):
            best = W[b, h, :n].topk(200).indices.sort().values
            assert torch.equal(kept[b, h].long(), best)
            assert torch.equal(k2[b, :, h], k[b, 500 - n + best, h]) and torch.equal(v2[b, :, h], v[b, 500 - n + best, h])


def test_python_refusals():
    need_gpu()
    case = case_of(12, [40, 30], 2, 64, 32, 10)
    cache, batch = case.cache(), case.batch()
    W, n = torch.rand(2, 2, 96, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    to = torch.from_numpy(case.target).cuda()
    kept = torch.zeros(2, 2, 10, dtype=torch.int32, device="cuda")
    ok = dict(cache=cache, batch=batch, W=W, new_lengths=n, budget=10)
    for bad in (dict(W=W.cpu()), dict(W=W.double()), dict(new_lengths=n.long()), dict(new_lengths=n[:1]), dict(budget=-1),
                dict(budget=2 ** 31), dict(first=-1), dict(to=to.long()), dict(to=to[:1]), dict(to=to.cpu()), dict(kept=kept[..., :9]),
                dict(kept=kept.float()), dict(to=to, W_to=W[0]), dict(workspace=torch.zeros(10 ** 6, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            cq.cqsa_cache_evict(**{**ok, **bad})
    for bad in (dict(budget=0), dict(first=6, recent=5), dict(W=W[..., :50]), dict(W_to=W), dict(to=to, W_to=W), dict(new_lengths=None),
                dict(workspace=torch.zeros(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(cq.CqsaError):
            cq.cqsa_cache_evict(**{**ok, **bad})
    before = cache.data.clone()
    cq.cqsa_cache_evict(**ok, to=to)
    rest = torch.ones(case.n_pages, dtype=torch.bool, device="cuda")
    rest[to[to >= 0].long()] = False
    assert torch.equal(cache.data[rest], before[rest]) and n.tolist() == [10, 10]


def test_strided_weights_another_stream_and_capture():
    need_gpu()
    say("evict captured")
    case = case_of(8, [150, 60], 2, 64, 32, 40)
    T = case.table.shape[1] * 32
    store = torch.rand(2, 4, T + 9, device="cuda")
    W = store[:, 1:3, 4:4 + T]
    before = W.cpu().numpy().copy()
    W_to = torch.full((2, 2, 40), 7.0, device="cuda")
    to = torch.from_numpy(case.target).cuda()
    kept = torch.zeros(2, 2, 40, dtype=torch.int32, device="cuda")
    new = torch.zeros(2, dtype=torch.int32, device="cuda")
    cache, batch = case.cache(), case.batch()
    space = cq.cqsa_cache_evict_workspace(cache, batch, 40, to)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    call = lambda: cq.cqsa_cache_evict(cache, batch, W, new, 40, 1, 5, to=to, W_to=W_to, kept=kept, workspace=space)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    with torch.cuda.graph(graph):
        call()
    data, kk, lens, Wn = moved(case, before, 40, 1, 5, case.target)
    for i in range(4):
        space.fill_(255 - i)
        kept.fill_(i)
        W_to.fill_(7.0)
        new.fill_(-1)
        for t in case.target[case.target >= 0]:
            cache.data[int(t)] = torch.from_numpy(case.data[t]).cuda()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(cache.data.cpu().numpy(), data) and np.array_equal(kept.cpu().numpy(), kk)
        assert np.array_equal(new.cpu().numpy(), lens) and same(W_to.cpu().numpy()[:, :, :40].copy(), Wn[:, :, :40].copy())


def test_attention_over_what_is_kept():
    """With a budget that keeps all that a query looks at, attention is as before."""
    need_gpu()
    say("evict attend")
    case = Case(9, [90], 1, 64, 32)
    case.fill_tokens()
    cache, batch = case.cache(), case.batch()
    q = torch.randn(1, 1, 2, 64, device="cuda")
    W = torch.zeros(1, 1, case.table.shape[1] * 32, device="cuda")
    lse = torch.zeros(1, 2, 1, device="cuda")
    o = torch.empty_like(q)
    cq.cqsa_cache_attend(cache, batch, q, o, lse)
    cq.cqsa_cache_weigh(cache, batch, q, lse, W)
    lengths = torch.zeros(1, dtype=torch.int32, device="cuda")
    cq.cqsa_cache_evict(cache, batch, W, lengths, 60)
    after = cq.CacheBatch(batch.pages, lengths)
    o2, lse2, W2 = torch.empty_like(q), torch.zeros_like(lse), torch.zeros_like(W)
    cq.cqsa_cache_attend(cache, after, q, o2, lse2)
    # what is gone is the rest of the weights' sum of 2 (over the two heads)
    share = W[0, 0, :60].double().sum() / 2
    mean = torch.exp((lse2 - lse).double()).mean()
    assert abs(float(mean - share)) < 64 * 2.0 ** -20
    assert float(share) > 0.6 and math.isfinite(float(share))
