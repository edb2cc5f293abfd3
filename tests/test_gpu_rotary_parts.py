"""Rotary positions between parts of one buffer.  Bounds as in tests/test_gpu_rotary.py."""
import numpy as np
import pytest
import torch

import paper_2604_20819_amd as cq
from tests.gpu_util import need_gpu
from tests.test_gpu_rotary import DT, held

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_from_heads_to_others_of_one_buffer(dtype):
    """Q and K of a buffer's first heads into its last ones; the rest of it stays."""
    need_gpu()
    B, L, d, sections = 2, 37, 96, (16, 24)
    g = np.random.Generator(np.random.PCG64(3))
    whole = torch.from_numpy(g.standard_normal((B, L, 13, d), dtype=np.float32)).to(DT[dtype])
    pos = torch.from_numpy(g.integers(0, 50000, (2, B, L)).astype(np.int32))
    w = whole.cuda()
    plan = cq.cqsa_rotary_plan(d, sections)
    cq.cqsa_rotary(plan, pos.cuda(), [w[:, :, :4], w[:, :, 4:6]], [w[:, :, 7:11], w[:, :, 11:]])
    held(w[:, :, 7:11], whole[:, :, :4], pos, dtype, sections=sections)
    held(w[:, :, 11:], whole[:, :, 4:6], pos, dtype, sections=sections)
    assert torch.equal(w[:, :, :7].cpu(), whole[:, :, :7])
