"""Rotary positions whose scale is far from 1, on the GPU, against 60 decimal digits.

Bound: the header's, 2^-32 + 2^-64 (1 + pos_scale) |pos| turns of a pair's angle, as radians times
the pair's |a| + |b|, and the arithmetic's 2^-21 of that (tests/test_gpu_rotary.py)."""
import decimal
import math

import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu
PI = decimal.Decimal("3.14159265358979323846264338327950288419716939937510582097494459")


def turns(pos, scale, theta, i, n):
    """The angle of pair i of n at a position, in turns without the whole ones."""
    with decimal.localcontext() as c:
        c.prec = 60
        f = decimal.Decimal(scale) * (-(decimal.Decimal(theta).ln() * i / n)).exp()
        return float((decimal.Decimal(int(pos)) * f / (2 * PI)) % 1)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 25.0, 1e4, 1e6])
@pytest.mark.parametrize("theta", [10000.0, 1e6])
def test_scaled_positions(scale, theta):
    need_gpu()
    d, n = 64, 32
    where = [0, 1, -1, 77, 4095, 2 ** 20 + 1, 123456789, -987654321, 2 ** 31 - 1, -2 ** 31]
    g = np.random.Generator(np.random.PCG64(int(theta)))
    x = g.standard_normal((1, len(where), 1, d), dtype=np.float32)
    plan = cq.cqsa_rotary_plan(d, (n,), theta=theta, pos_scale=(scale,))
    y = torch.empty(x.shape, device="cuda")
    cq.cqsa_rotary(plan, torch.tensor([[where]], dtype=torch.int32).cuda(), torch.from_numpy(x).cuda(), y)
    got = y.cpu().double().numpy()[0, :, 0]
    for k, p in enumerate(where):
        angle = 2 * math.pi * np.array([turns(p, scale, theta, i, n) for i in range(n)])
        a, b = x[0, k, 0, :n].astype(np.float64), x[0, k, 0, n:].astype(np.float64)
        off = 2 * math.pi * (2.0 ** -32 + 2.0 ** -64 * (1 + scale) * abs(p)) + 2.0 ** -21
        bound = (np.abs(a) + np.abs(b)) * off
        assert (np.abs(got[k, :n] - (a * np.cos(angle) - b * np.sin(angle))) <= bound).all(), p
        assert (np.abs(got[k, n:] - (b * np.cos(angle) + a * np.sin(angle))) <= bound).all(), p
