"""The kernels of the cached tokens' attention weights on the CPU: their own source, every lane a fiber, in
buffers of exact sizes under the address sanitizer, each call twice in other orders of its waves and work groups,
and every weight against a sum in 64 bits (tests/lanes; no GPU)."""
import os
import re
import subprocess

import pytest

from paper_2604_20819_amd import build
from tests.op_util import WEIGH_LOOPS

HERE = os.path.join(os.path.dirname(os.path.abspath(__file__)), "lanes")


@pytest.fixture(scope="module")
def weigh(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("lanes") / "weigh")
    clang = os.path.join(os.path.dirname(os.path.realpath(build.hipcc())), "..", "lib", "llvm", "bin", "clang++")
    cmd = [clang, "-std=c++17", "-O1", "-g1", "-w", "-D__HIPCC__",
           # the kernels ask for their loops unrolled, which here only takes long to compile
           "-mllvm", "-pragma-unroll-threshold=1", "-mllvm", "-unroll-threshold=1", "-fno-vectorize", "-fno-slp-vectorize",
           "-fsanitize=address", "-mllvm", "-asan-stack=0",
           "-I", HERE, "-I", build.CSRC, "-I", build.INCLUDE,
           "-x", "c++", os.path.join(HERE, "weigh.cpp"), "-x", "c++", os.path.join(HERE, "lanes.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(**kw):
        """The launch that the call took: row_groups, resident, waves, tiles, splits, and a_wave, how many of its
        tiles a wave goes through."""
        args = [f"{k}={','.join(map(str, v)) if isinstance(v, (list, tuple)) else int(v)}" for k, v in kw.items()]
        r = subprocess.run([exe] + args, capture_output=True, text=True, timeout=200,
                           env={**os.environ, "ASAN_OPTIONS": "detect_leaks=0"})
        assert r.returncode == 0, (args, r.stdout[-2000:], r.stderr[-3000:])
        return {k: int(v) for k, v in re.findall(r"(\w+) (\d+)", r.stdout.splitlines()[0])}

    return run


# sequences of up to 400 tokens, each with 64 rows, some with fewer tokens than that
LENGTHS = [int(400 * ((b * 0.6180339887) % 1.0)) if b else 400 for b in range(0, 32, 3)]
TYPES = [(0, 1), (1, 0), (2, 1), (2, 0)]  # dtype, in place


def test_more_rows_than_tokens(weigh):
    """64 rows of 8 heads to one over many short sequences: the rows in 4 parts, of which causal masks leave some
    without rows, and sequences shorter than their rows."""
    p = weigh(L=64, H=1, G=8, d=32, lens=LENGTHS)
    assert p["row_groups"] == 0 and not p["resident"] and p["splits"] == 4
    p = weigh(L=64, H=8, G=8, d=32, lens=[400, 27, 0], holes=1)
    assert p["splits"] == 4
    weigh(L=64, H=1, G=8, d=32, lens=[63, 64, 65, 1], causal=0, counted=1)
    weigh(L=64, H=2, G=8, d=32, lens=[200, 16, 130], new=[64, 7, 40], page_log2=5)


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_streamed_rows(weigh, dtype):
    for d, L, G, lens in ((64, 45, 3, [150, 20, 0]), (128, 33, 5, [70, 33]), (224, 70, 2, [100, 65])):
        p = weigh(dtype=dtype, d=d, L=L, G=G, lens=lens, page_log2=5, holes=1, in_place=d == 64, seed=d)
        assert p["row_groups"] == 0 and not p["resident"]


def test_streamed_rows_that_fold(weigh):
    """A split of more than 1024 rows, whose sums pass through a total."""
    p = weigh(L=2304, H=1, G=1, d=32, lens=[70], max_len=2 ** 18, prior=0)
    assert p["row_groups"] == 0 and not p["resident"] and 2304 / p["splits"] > 1024


@pytest.mark.parametrize("dtype,in_place", TYPES)
def test_few_rows_over_many_tiles(weigh, dtype, in_place):
    """Waves that go through several tiles of 32 tokens, the next one's keys and prior on their way; more than 64,
    whose pages they read again."""
    for d, L, G, lens, tiles in ((32, 1, 1, [9000, 700], 1), (128, 5, 3, [700, 1025, 31], 2), (96, 2, 8, [500, 64], 1)):
        p = weigh(dtype=dtype, d=d, L=L, G=G, lens=lens, tiles=tiles, in_place=in_place, holes=1, page_log2=5)
        assert p["row_groups"] == (1 if L * G <= 16 else 2) and p["a_wave"] >= (65 if d == 32 else 4)


@pytest.mark.parametrize("dtype,in_place", TYPES)
def test_resident_rows_over_many_tiles(weigh, dtype, in_place):
    """Work groups whose rows stay, and that go on to further tiles of 64 tokens a wave."""
    for d, L, G, lens in ((32, 9, 5, [900, 300]), (96, 33, 1, [600, 33]), (256, 10, 4, [1050])):
        p = weigh(dtype=dtype, d=d, L=L, G=G, lens=lens, tiles=1, in_place=in_place, holes=1, page_log2=5)
        assert p["resident"] and p["a_wave"] >= 3


@pytest.mark.parametrize("B,H,G,L,d,dtype,n", WEIGH_LOOPS)
def test_launches_of_several_tiles(weigh, B, H, G, L, d, dtype, n):
    """The launches of tests/test_gpu_cache_weigh.py's test of such waves."""
    p = weigh(lens=[n] * B, H=H, G=G, L=L, d=d, dtype=["f32", "f16", "bf16"].index(dtype), dry=1)
    assert (p["row_groups"] > 0 or p["resident"]) and p["a_wave"] >= (65 if n > 50000 else 2 if p["resident"] else 3)
