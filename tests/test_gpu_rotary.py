"""Rotary positions on the GPU against extended precision (oracle.rotary).

Bound of an element: its pair's |a| + |b| times 2^-21, and half a step of the
result's type.  The sine and cosine are off by under 2^-22: the reduced angle
(at most pi / 4) is rounded twice (2 x 2^-24 x .79), the position's fixed-point
angle is off by 2^-32 turns, the sums end with terms under 2e-9 and round a
value of at most 1 twice.  The two products and their sum round by at most
2^-23 (|a| + |b|) more.
"""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import rotary as orot
from paper_2604_20819_amd import synth
from tests.gpu_util import need_gpu, say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {k: torch.finfo(v).eps / 2 for k, v in DT.items()}


def inputs(seed, dtype, B, L, heads, d, far, axes):
    g = np.random.Generator(np.random.PCG64(seed))
    xs = [torch.from_numpy(g.standard_normal((B, L, h, d), dtype=np.float32)).to(DT[dtype]) for h in heads]
    pos = g.integers(-far, far, (axes, B, L), dtype=np.int64).clip(-2 ** 31, 2 ** 31 - 1).astype(np.int32)
    return xs, torch.from_numpy(pos)


def held(got, x, pos, dtype, **kw):
    want, size = orot.rotate(synth.as_f64(x), pos.numpy(), **kw)
    err = np.abs(got.cpu().double().numpy() - want)
    assert got.dtype == DT[dtype]
    bound = size * 2.0 ** -21
    bound = bound + HALF_STEP[dtype] * (np.abs(want) + bound)
    if dtype == "f16":
        bound += 2.0 ** -25  # half a step below its normal range
    assert (err <= bound).all(), (err - bound).max()
    still = 2 * sum(kw["sections"])
    assert np.array_equal(got.cpu().double().numpy()[..., still:], synth.as_f64(x)[..., still:])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("d,sections,spectrum,dealt", [
    (32, (8,), "shared", False), (128, (16, 24, 24), "shared", False),
    (128, (22, 21, 21), "per_axis", False), (96, (24, 16), "shared", True),
    (256, (32, 32, 33, 31), "per_axis", True), (160, (3, 1, 60), "shared", True)])
def test_against_extended_precision(dtype, pairs, d, sections, spectrum, dealt):
    need_gpu()
    B, L, heads = 2, 37, (5, 2)
    kw = dict(sections=sections, spectrum=spectrum, dealt=dealt, pairs=pairs, theta=10000.0)
    xs, pos = inputs(d + len(sections), dtype, B, L, heads, d, 2 ** 20, len(sections))
    say("rotary", dtype, pairs, d, sections, spectrum, dealt)
    plan = cq.cqsa_rotary_plan(d, sections, pairs=pairs, spectrum=spectrum, dealt=dealt)
    for inverse in (False, True):
        ys = [torch.full_like(x, 7.0, device="cuda") for x in xs]
        cq.cqsa_rotary(plan, pos.cuda(), [x.cuda() for x in xs], ys, inverse=inverse)
        for x, y in zip(xs, ys):
            held(y, x, pos, dtype, inverse=inverse, **kw)


@pytest.mark.parametrize("B,L,heads", [(1, 1, (1,)), (3, 1, (32, 8)), (1, 1000, (1, 1)), (64, 1, (7,)),
                                       (1, 4099, (3, 17))])
def test_sizes(B, L, heads):
    need_gpu()
    d, sections = 64, (8, 12, 12)
    xs, pos = inputs(L, "bf16", B, L, heads, d, 5000, 3)
    say("rotary sizes", B, L, heads)
    plan = cq.cqsa_rotary_plan(d, sections)
    ys = [torch.empty_like(x, device="cuda") for x in xs]
    cq.cqsa_rotary(plan, pos.cuda(), [x.cuda() for x in xs], ys)
    for x, y in zip(xs, ys):
        held(y, x, pos, "bf16", sections=sections)


def test_far_and_negative_positions():
    """Positions at both ends of int32, and the scale and theta of an axis."""
    need_gpu()
    d, sections = 64, (16, 16)
    g = np.random.Generator(np.random.PCG64(5))
    x = torch.from_numpy(g.standard_normal((1, 6, 2, d), dtype=np.float32))
    pos = torch.tensor([[[-2 ** 31, 2 ** 31 - 1, -1, 0, 123456789, -987654321]]] * 2, dtype=torch.int32)
    plan = cq.cqsa_rotary_plan(d, sections, theta=500000.0, pos_scale=(0.25, 1.0))
    y = torch.empty_like(x, device="cuda")
    cq.cqsa_rotary(plan, pos.cuda(), x.cuda(), y)
    held(y, x, pos, "f32", sections=sections, theta=500000.0, pos_scale=(0.25, 1.0))


def test_in_place_and_strided():
    """Q and K as parts of one projection, turned where they are: the rest stays."""
    need_gpu()
    B, L, Hq, Hk, d, sections = 2, 19, 6, 2, 128, (16, 16, 16)
    g = np.random.Generator(np.random.PCG64(9))
    whole = torch.from_numpy(g.standard_normal((B, L, Hq + 2 * Hk, d), dtype=np.float32)).bfloat16()
    pos = torch.from_numpy(g.integers(0, 3000, (3, B, L)).astype(np.int32))
    w = whole.cuda()
    q, k = w[:, :, :Hq], w[:, :, Hq:Hq + Hk]
    plan = cq.cqsa_rotary_plan(d, sections)
    cq.cqsa_rotary(plan, pos.cuda(), [q, k])
    held(q, whole[:, :, :Hq], pos, "bf16", sections=sections)
    held(k, whole[:, :, Hq:Hq + Hk], pos, "bf16", sections=sections)
    assert torch.equal(w[:, :, Hq + Hk:].cpu(), whole[:, :, Hq + Hk:])
    # heads before tokens, read through its strides and through a broadcast batch
    t = whole.cuda().transpose(1, 2).contiguous().transpose(1, 2)
    y = torch.empty((B, L, Hq + 2 * Hk, d), dtype=torch.bfloat16, device="cuda")
    cq.cqsa_rotary(plan, pos.cuda(), t, y)
    held(y, whole, pos, "bf16", sections=sections)
    one = whole[:1].expand(B, -1, -1, -1)
    cq.cqsa_rotary(plan, pos.cuda(), one.cuda()[:1].expand(B, -1, -1, -1), y)
    held(y, one, pos, "bf16", sections=sections)


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_gradient(pairs):
    """inverse=True is the gradient: <R x, g> = <x, R' g>, and differences of the loss
    <R x, g> (linear in x, so a step of 1 is exact up to rounding) give R' g."""
    need_gpu()
    B, L, H, d, sections = 1, 5, 2, 64, (8, 8)
    gen = np.random.Generator(np.random.PCG64(11))
    x, g = (torch.from_numpy(gen.standard_normal((B, L, H, d), dtype=np.float32)).cuda() for _ in range(2))
    pos = torch.from_numpy(gen.integers(0, 100000, (2, B, L)).astype(np.int32)).cuda()
    plan = cq.cqsa_rotary_plan(d, sections, pairs=pairs)

    def turned(v, inverse=False):
        y = torch.empty_like(v)
        cq.cqsa_rotary(plan, pos, v, y, inverse=inverse)
        return y

    grad = turned(g, inverse=True)
    a, b = (turned(x).double() * g).sum(), (x.double() * grad).sum()
    assert abs(a - b) <= 2.0 ** -20 * (x.double().abs() * g.abs()).sum() * 2
    base = (turned(x).double() * g).sum()
    for at in [(0, 0, 0, 0), (0, 3, 1, 7), (0, 4, 0, 33), (0, 2, 1, 63)]:
        z = x.clone()
        z[at] += 1.0
        diff = (turned(z).double() * g).sum() - base
        # two losses, each off by 2^-21 of the sum of the pairs' sizes
        assert abs(diff - grad[at].double()) <= 2.0 ** -19 * (x.abs().double() + 1).sum() * g.abs().max()


def test_empty_calls_write_nothing():
    need_gpu()
    plan = cq.cqsa_rotary_plan(64)
    for shape in [(0, 4, 2, 64), (2, 0, 2, 64), (2, 4, 0, 64)]:
        x = torch.empty(shape, device="cuda")
        cq.cqsa_rotary(plan, torch.zeros((1,) + shape[:2], dtype=torch.int32, device="cuda"), x, torch.empty_like(x))
    torch.cuda.synchronize()


def test_captured_and_on_another_stream():
    need_gpu()
    d, sections = 64, (16, 16)
    xs, pos = inputs(3, "bf16", 1, 300, (4,), d, 1000, 2)
    plan = cq.cqsa_rotary_plan(d, sections)
    x, p = xs[0].cuda(), pos.cuda()
    y = torch.empty_like(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cq.cqsa_rotary(plan, p, x, y)
    for k in range(4):
        fresh = (xs[0] * (k + 1)).to(torch.bfloat16)
        x.copy_(fresh)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        held(y, fresh, pos, "bf16", sections=sections)
    y.zero_()
    torch.cuda.synchronize()
    cq.cqsa_rotary(plan, p, x, y, stream=s.cuda_stream)
    s.synchronize()
    held(y, fresh, pos, "bf16", sections=sections)
