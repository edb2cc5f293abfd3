"""The operators' compiled kernels: no register spill under a branch's partial exec mask
(tests/test_kernel_asm.py says why), and no packed fp32 arithmetic (CPU only)."""
import concurrent.futures
import re

import pytest

from paper_2604_20819_amd import build

SOURCES = ["rotary.hip", "cache_quant.hip", "cache_attend.hip", "cache_attend_many.hip"]


@pytest.fixture(scope="module")
def asm():
    with concurrent.futures.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(build.device_asm, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_no_spill_under_a_partial_exec_mask(src, asm):
    assert src in build.SOURCES and ".amdhsa_kernel" in asm[src]
    assert build.masked_spill_stores(asm[src]) == {}


@pytest.mark.parametrize("src", SOURCES)
def test_no_packed_fp32(src, asm):
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", asm[src])
