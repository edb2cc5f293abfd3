"""cqsa_draft_verify against the float64 oracle: every token exactly.

A drawn token is where a sum in 64 bits passes a share of it.  The oracle says how near the share is to a border:
V sums round by less than V 2^-53 of the whole, and inputs are made so that none is that near.
"""
import math

import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import bounded as ob
from tests.gpu_util import need_gpu, say
from tests.op_util import DT

pytestmark = pytest.mark.gpu


def inputs(seed, B, K, V, dtype, draft=True, peak=3.0, near=0.5):
    g = np.random.Generator(np.random.PCG64(seed))
    x = g.standard_normal((B, K + 1, V)) * peak
    y = x[:, :K] + near * g.standard_normal((B, K, V))

    def soft(z):
        z = np.exp(z - z.max(-1, keepdims=True))
        return torch.from_numpy((z / z.sum(-1, keepdims=True)).astype(np.float32)).to(DT[dtype])

    p, q = soft(x), soft(y)
    noise = -np.log(g.exponential(size=(B, K, V)))
    tokens = torch.from_numpy((y + noise).argmax(-1).astype(np.int32))
    u = torch.from_numpy(g.random((B, K + 1), dtype=np.float32))
    return p, q if draft else None, tokens, u


def run(p, q, tokens, u, counts=None, lengths=None, alias=False, device=True):
    B, K, V = p.shape[0], p.shape[1] - 1, p.shape[2]
    cuda = lambda t: None if t is None else t.cuda() if t.is_contiguous() else t
    out = torch.full((B, K + 1), 77, dtype=torch.int32, device="cuda")
    n_out = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    new = None if lengths is None else ln if alias else torch.full((B,), 77, dtype=torch.int32, device="cuda")
    cn = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
    cq.cqsa_draft_verify(cuda(p), cuda(q), cuda(tokens), cuda(u), out, n_out, counts=cn, lengths=ln, new_lengths=new)
    got = out.cpu().numpy(), n_out.cpu().numpy(), None if new is None else new.cpu().numpy()
    P, Q = p.double().cpu().numpy(), None if q is None else q.double().cpu().numpy()
    for b in range(B):
        o, n, l, near = ob.verify(P[b], None if Q is None else Q[b], tokens[b].cpu().numpy(), K if counts is None else counts[b],
                                  u[b].double().cpu().numpy(), None if lengths is None else lengths[b])
        assert near > V * 2.0 ** -53 or near == 0.0, "an input on a border"
        assert n == got[1][b] and np.array_equal(o, got[0][b]), (b, o, got[0][b])
        if l is not None:
            assert l == got[2][b]
    return got


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,K,V", [(1, 1, 1), (3, 2, 2), (2, 4, 63), (5, 3, 64), (4, 5, 65), (3, 1, 1000), (2, 8, 4097),
                                   (2, 3, 32003), (1, 2, 131072), (70, 2, 515), (300, 3, 129), (2, 64, 300)])
def test_tokens(B, K, V, draft, dtype):
    need_gpu()
    say("verify", B, K, V, draft, dtype)
    p, q, tokens, u = inputs(B * 1000 + K * 7 + V, B, K, V, dtype, draft)
    g = np.random.Generator(np.random.PCG64(V))
    run(p, q, tokens, u, lengths=[int(x) for x in g.integers(K + 1, 100, B)])
    run(p, q, tokens, u, counts=[int(x) for x in g.integers(-1, K + 2, B)], lengths=[int(x) for x in g.integers(0, 3, B)], alias=True)


@pytest.mark.parametrize("B,K,V,dtype,draft", [
    (130, 1, 70001, "f32", True), (130, 1, 70001, "bf16", False), (129, 2, 100003, "f32", False), (129, 1, 100003, "f16", True),
    (17, 2, 131073, "f32", True), (18, 1, 200003, "bf16", True), (20, 2, 200003, "f32", False), (19, 2, 262144, "f32", True),
    (19, 2, 262144, "bf16", False), (3, 1, 1048577, "f16", True), (128, 1, 600001, "bf16", False)])
def test_large_vocabularies(B, K, V, dtype, draft):
    """Pieces of the vocabulary that take several loads of a wave, many pieces a wave, and more elements of the drawn
    piece a thread than it holds: shares of the sum near 0 and 1 too, strange probabilities in some loads of a piece
    and not in others, refused tokens anywhere."""
    need_gpu()
    say("verify large", B, K, V, dtype, draft)
    p, q, tokens, u = inputs(V + B, B, K, V, dtype, draft, peak=1.0)
    g = np.random.Generator(np.random.PCG64(B))
    bad = torch.tensor([math.nan, math.inf, -math.inf, -1.0, -0.0])
    for b in range(0, B, 3):
        at = torch.from_numpy(g.integers(0, V, 40))
        p[b, :, at] = bad[torch.arange(40) % 5].to(p.dtype)
        if draft:
            q[b, :, at.roll(1)] = bad[(torch.arange(40) + 2) % 5].to(p.dtype)
    if not draft:
        tokens = torch.from_numpy(g.integers(0, V, (B, K), dtype=np.int32))
    u[1::8, K] = torch.linspace(1e-7, 1e-4, len(u[1::8]))
    u[2::8, K] = 1 - 2.0 ** -24 * torch.arange(1, len(u[2::8]) + 1)
    u[::2, 0] = 0.9999
    run(p, q, tokens, u, counts=[int(x) for x in g.integers(0, K + 1, B)], lengths=[int(x) for x in g.integers(K + 1, 100, B)])


def test_draws_over_the_whole_range():
    """One row, many draws: u = 0 is the first token with any probability, near 1 the last."""
    need_gpu()
    say("verify draws")
    V = 3001
    p, q, tokens, _ = inputs(1, 1, 1, V, "f32", peak=1.0)
    p[0, :, :5] = 0
    p[0, :, -5:] = 0
    n = 200
    u = torch.rand(n, 2, generator=torch.Generator().manual_seed(3))
    u[0, 1], u[1, 1], u[2, 1], u[3, 1] = 0.0, float(np.nextafter(np.float32(1), np.float32(0))), 1.0, math.nan
    u[:, 0] = torch.where(torch.arange(n) % 2 == 0, 0.0, 0.9999)
    P, Q, t = (x.expand(n, -1, -1).contiguous() if x.dim() == 3 else x.expand(n, -1).contiguous() for x in (p, q, tokens))
    u0 = u.clone()
    u0[:4, 1] = 0.5
    run(P, Q, t, u0)
    out = torch.zeros(n, 2, dtype=torch.int32, device="cuda")
    n_out = torch.zeros(n, dtype=torch.int32, device="cuda")
    cq.cqsa_draft_verify(P.cuda(), None, t.cuda(), u.cuda(), out, n_out, counts=torch.zeros(n, dtype=torch.int32, device="cuda"))
    assert out[0, 0] == 5 and out[3, 0] == 5 and out[2, 0] == V - 6 and out[1, 0] <= V - 6
    assert (n_out == 1).all() and (out[:, 1] == -1).all()


def test_distribution_is_the_targets():
    """Over many given numbers the first token's frequencies are the target's."""
    need_gpu()
    say("verify distribution")
    V, n = 7, 200000
    g = torch.Generator().manual_seed(11)
    p = torch.softmax(torch.randn(1, 2, V, generator=g), -1)
    q = torch.softmax(torch.randn(1, 1, V, generator=g), -1)
    x = torch.multinomial(q[0, 0], n, replacement=True, generator=g).int()[:, None].contiguous()
    u = torch.rand(n, 2, generator=g)
    out = torch.zeros(n, 2, dtype=torch.int32, device="cuda")
    n_out = torch.zeros(n, dtype=torch.int32, device="cuda")
    cq.cqsa_draft_verify(p.cuda().expand(n, -1, -1), q.cuda().expand(n, -1, -1), x.cuda(), u.cuda(), out, n_out)
    share = torch.bincount(out[:, 0].long(), minlength=V).double().cpu() / n
    # five standard deviations of a frequency at most
    assert (share - p[0, 0].double()).abs().max() < 5 * 0.5 / math.sqrt(n)


def test_equal_distributions_accept_all():
    need_gpu()
    say("verify equal")
    p, _, tokens, u = inputs(2, 6, 4, 500, "bf16")
    q = p[:, :4].clone()
    tokens = torch.multinomial(q.float().reshape(-1, 500), 1).reshape(6, 4).int()
    out, n_out, _ = run(p, q, tokens, u)
    assert (n_out == 5).all()


def test_rest_of_nothing_is_the_target():
    """p below q wherever p has any, which rounding can leave: the draw is from p."""
    need_gpu()
    say("verify rest")
    p, q, tokens, u = inputs(3, 3, 1, 700, "f32")
    q[:] = 2 * p[:, :1]
    u[:, 0] = 0.75
    out, n_out, _ = run(p, q, tokens, u)
    assert (n_out == 1).all()
    p, _, _, u = inputs(3, 2, 1, 40, "f32")
    p.zero_()
    p[:, :, 9] = 0.5
    t = torch.full((2, 1), 9, dtype=torch.int32)
    u[:, 0] = 0.5
    run(p, None, t, u)  # all that there is was refused
    p[:, :, 9] = 3.0
    run(p, None, t, u)


def test_numbers_that_are_none_and_tokens_outside():
    need_gpu()
    say("verify strange")
    p, q, tokens, u = inputs(4, 8, 3, 300, "f32")
    bad = torch.tensor([math.nan, math.inf, -math.inf, -1.0, -0.0])
    for b in range(8):
        p[b, :, b:250:17] = bad[b % 5]
        q[b, :, b + 3:250:13] = bad[(b + 2) % 5]
    tokens[0, 0], tokens[1, 1], tokens[2, 0], tokens[3, 0] = -1, 300, 2 ** 31 - 1, -2 ** 31
    u[4, 1], u[5, 0], u[6, 2] = math.nan, math.nan, 1.5
    run(p, q, tokens, u)
    run(p, None, tokens, u)
    p[:] = math.nan  # nothing to draw from
    out, n_out, _ = run(p, q, tokens, u)
    assert (out == -1).all() and (n_out == 1).all()


def test_subnormal_probabilities():
    need_gpu()
    say("verify subnormal")
    p, q, tokens, u = inputs(7, 3, 2, 400, "f32")
    for f in (1e-38, 1e-41):
        a, b = (p.double() * f).float(), (q.double() * f).float()
        run(a, b, tokens, u)
        run(a, None, tokens, u)


def test_rows_far_apart():
    """Rows whose elements lie past 2^31."""
    need_gpu()
    say("verify far")
    V, far = 1001, 2 ** 31 + 10 ** 6
    p, q, tokens, u = inputs(8, 2, 1, V, "bf16")
    store = torch.empty(far + 3 * 10 ** 6, dtype=torch.bfloat16, device="cuda")
    P = store.as_strided((2, 2, V), (far, 10 ** 5 + 1, 1))
    Q = store.as_strided((2, 1, V), (far, V, 1), 10 ** 6 + 7)
    P.copy_(p)
    Q.copy_(q)
    run(P, Q, tokens, u)
    P = store.as_strided((2, 2, V), (10 ** 6, far, 1))
    P.copy_(p)
    run(P, None, tokens, u)


def test_python_refusals():
    need_gpu()
    p, q, tokens, u = (x.cuda() for x in inputs(9, 2, 2, 64, "f32"))
    out, n = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(target=p, draft=q, tokens=tokens, u=u, out=out, n_out=n)
    for bad in (dict(target=p.cpu()), dict(target=p.double()), dict(target=p[0]), dict(draft=q.transpose(1, 2)), dict(draft=q.cpu()),
                dict(tokens=tokens.long()), dict(tokens=tokens[:1]), dict(u=u.double()), dict(u=u[:, :2]), dict(out=out[:, :2]),
                dict(n_out=n.cpu()), dict(counts=n.float()), dict(workspace=torch.zeros(64, dtype=torch.uint8)),
                dict(lengths=n, new_lengths=n.long())):
        with pytest.raises(ValueError):
            cq.cqsa_draft_verify(**{**ok, **bad})
    for bad in (dict(lengths=n), dict(draft=q.half()), dict(draft=p), dict(out=tokens.new_zeros(2, 3), n_out=None)):
        with pytest.raises(cq.CqsaError):
            cq.cqsa_draft_verify(**{**ok, **bad})
    cq.cqsa_draft_verify(**ok)


def test_missing_arguments_are_named():
    need_gpu()
    p, q, tokens, u = (x.cuda() for x in inputs(9, 2, 2, 64, "f32"))
    out, n = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(target=p, draft=q, tokens=tokens, u=u, out=out, n_out=n)
    for name in ("target", "u"):
        with pytest.raises(ValueError, match=name + " must"):
            cq.cqsa_draft_verify(**{**ok, name: None})
    for name in ("tokens", "out", "n_out"):
        with pytest.raises(cq.CqsaError, match=name + " is NULL"):
            cq.cqsa_draft_verify(**{**ok, name: None})


def test_odd_strides_and_alignment():
    """Rows that begin at any element, broadcast targets, rows that lie apart."""
    need_gpu()
    say("verify strides")
    for dtype in ("f32", "f16", "bf16"):
        p, q, tokens, u = inputs(5, 3, 2, 333, dtype)
        for shift in (1, 3, 7):
            big = torch.full((3, 5, 400), 9.0, dtype=DT[dtype], device="cuda")
            P = big[:, 1:4, shift:shift + 333]
            P.copy_(p)
            big2 = torch.full((3, 2, 341), 9.0, dtype=DT[dtype], device="cuda")
            Q = big2[:, :, 8 - shift:341 - shift]
            Q.copy_(q)
            run(P, Q, tokens, u)
        run(p[:1].cuda().expand(3, -1, -1), q[:1].cuda().expand(3, -1, -1), tokens, u)


def test_captured_and_on_another_stream():
    need_gpu()
    say("verify captured")
    for B, V in ((2, 50001), (40, 2000)):
        p, q, tokens, u = (x.cuda() for x in inputs(6, B, 3, V, "bf16"))
        out = torch.zeros(B, 4, dtype=torch.int32, device="cuda")
        n_out = torch.zeros(B, dtype=torch.int32, device="cuda")
        space = cq.cqsa_draft_verify_workspace(p, q)
        call = lambda: cq.cqsa_draft_verify(p, q, tokens, u, out, n_out, workspace=space)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for i in range(4):
            u.copy_(torch.rand(B, 4, generator=torch.Generator().manual_seed(i)))
            if space is not None:
                space.fill_(255 - i)
            out.fill_(55)
            graph.replay()
            a, b = out.clone(), n_out.clone()
            call()
            torch.cuda.synchronize()
            assert torch.equal(a, out) and torch.equal(b, n_out)
        got = run(p.cpu(), q.cpu(), tokens.cpu(), u.cpu())
        assert np.array_equal(got[0], out.cpu().numpy())
