"""Attention over the 4-bit cache on the GPU: weights that all round the same way.

Bound: values that do not differ between tokens come back as they are.  With
weights w' as the product takes them, O = sum w' v / sum w' = v whatever their
rounding, if the same w' are summed; fp32 sums of n <= 2048 terms are off by at
most n 2^-24 = 2^-13 each, under half of half a step (2^-9 for bf16 at the least),
so the result's rounding gives v itself.  LSE: as tests/test_gpu_cache_attend.py.
"""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from oracle import cache4 as o4
from tests.gpu_util import need_gpu, say
from tests.op_util import DT, Case
from tests.test_gpu_cache_attend import bounded, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kind,n,causal", [("few", 1, True), ("two", 40, True), ("two", 15, False),
                                           ("many", 70, True), ("many", 33, False)])
def test_alike_values_come_back(dtype, d, kind, n, causal):
    """One token of each 32 has the row's largest score, the others weigh .50176, which bf16 rounds
    down to .5: a sum of weights that are not the product's is off by 2^-8 of itself."""
    need_gpu()
    lens, G = (1999, 64, 777), 4
    case = Case(d + n, lens, 1, d, 64)
    value = np.resize([1.5, 3.0, -6.0, 1.0, 0.5], d)
    for b, m in enumerate(lens):
        k = np.zeros((m, 1, d))
        k[np.arange(m) % 32 != 0, 0, 0] = 1.0
        p, t = case.slots(b, 0, m)
        o4.write(case.data, 64, k, np.broadcast_to(value, k.shape), p, t)
    q = torch.zeros((3, n, G, d), dtype=DT[dtype])
    q[..., 0] = -1.0
    scale = float(np.float32(-np.log(0.50176)))
    say("attend alike", dtype, d, kind, n, causal)
    O, LSE = torch.full_like(q, 9.0, device="cuda"), torch.full((3, G, n), 9.0, device="cuda")
    cq.cqsa_cache_attend(case.cache(), bounded(case, kind), q.cuda(), O, LSE, causal=causal, scale=scale)
    want = torch.from_numpy(value).expand(3, n, G, d).clone()
    for b, m in enumerate(lens):  # causal rows before position 0 see nothing
        want[b, :max(n - m, 0) if causal else 0] = 0
    # fp32: half a step is 2^-24, the sums' own error counts; fp16: half a step of 2^-11 and the sums' up to 2^-12
    off, most = (O.cpu().double() - want).abs(), {"f32": 2.0 ** -12, "f16": 2.0 ** -10, "bf16": 0.0}[dtype]
    worst = (off - most * want.abs()).max().item()
    assert worst <= 0, worst
    for b, m in enumerate(lens):
        wl = reference(case, q[b].double().numpy(), b, m, causal, scale)[1]
        e = scale * (2.0 ** -20 + d * 2.0 ** -23)
        got, none = LSE[b].t().cpu().double().numpy(), np.isneginf(wl)
        assert np.array_equal(np.isneginf(got), none)
        off = np.abs(got[~none] - wl[~none])
        assert (off <= e + 2.0 ** -22 * (np.abs(wl[~none]) + 8)).all(), off.max()


@pytest.mark.parametrize("dtype,parts", [("bf16", 2.0 ** -16), ("f16", 2.0 ** -16), ("f32", 2.0 ** -22)])
@pytest.mark.parametrize("d", [64, 160])
def test_values_that_cancel(dtype, parts, d):
    """Few rows: values of both signs and weights nearly alike, so that the result is far below the
    weights' rounding.  Bound: 2 e + parts + n 2^-23 of the weights' sum of |v| (e the scores' error) and
    half a step, as in tests/test_gpu_cache_attend.py, with the bits that two (fp32: three) parts leave."""
    need_gpu()
    lens, G = (2, 3, 4, 9, 32, 33, 100, 257), 4
    case = Case(d, lens, 1, d, 32)
    for b, m in enumerate(lens):
        k = case.g.standard_normal((m, 1, d))
        v = np.where(np.arange(m) % 2, -1.0, 1.0)[:, None, None] * np.resize([1.0, 1.5, 3.0], d)
        p, t = case.slots(b, 0, m)
        o4.write(case.data, 32, k, v, p, t)
    q = (torch.from_numpy(case.g.standard_normal((len(lens), 1, G, d))) / 64).to(DT[dtype])
    say("attend cancel", dtype, d)
    x = cq.cqsa_cache_attend_launch(case.cache(), bounded(case, "few"), q.cuda())
    assert (x.many, x.rows) == (0, 16)
    O = torch.full_like(q, 9.0, device="cuda")
    cq.cqsa_cache_attend(case.cache(), bounded(case, "few"), q.cuda(), O)
    for b, m in enumerate(lens):
        wo, _, absv, big = reference(case, q[b].double().numpy(), b, m, True)
        e = big * (2.0 ** -20 + d * 2.0 ** -23)
        bound = (2 * e[..., None] + parts + m * 2.0 ** -23) * absv
        bound = bound + torch.finfo(DT[dtype]).eps / 2 * (np.abs(wo) + bound) + (2.0 ** -25 if dtype == "f16" else 0)
        off = np.abs(O[b].cpu().double().numpy() - wo)
        assert (off <= bound).all(), (m, (off - bound).max())
