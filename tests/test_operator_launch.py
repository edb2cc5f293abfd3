"""How attention over the 4-bit cache is launched, by its sizes alone (no GPU)."""
import ctypes

import pytest

import paper_2604_20819_amd as cq
from tests.test_operator_args import PTR, batch, cache, refused, view


def launch(c, b, q):
    out = cq.cqsa_attend_launch(7, 7, 7, 7)
    assert cq.lib().cqsa_cache_attend_launch(c, b, q, out) == 0, cq.lib().cqsa_last_error()
    return out


def long_batch(B=1, max_len=1 << 20, **kw):
    pages = -(-max_len // 64)
    return batch(B=B, max_pages=pages, pages_stride=pages, max_len=max_len, **kw)


@pytest.mark.parametrize("dtype", [cq.CQSA_BF16, cq.CQSA_F16, cq.CQSA_F32])
@pytest.mark.parametrize("d", [32, 96, 128, 160, 256])
def test_workspace_goes_by_the_splits(dtype, d):
    n = ctypes.c_uint64()
    for B, H, G, L, length in ((1, 1, 1, 1, 100), (1, 8, 2, 1, 1 << 20), (64, 8, 4, 1, 1 << 14), (1, 4, 4, 4096, 1 << 15),
                               (200, 1, 1, 1, 1000), (2, 2, 2, 20, 1 << 17), (64, 4, 1, 100, 200)):
        c, b, q = cache(H=H, d=d), long_batch(B, length), view(B=B, L=L, H=H * G, d=d, dtype=dtype)
        x = launch(c, b, q)
        assert cq.lib().cqsa_cache_attend_workspace(c, b, q, n) == 0
        assert n.value == (B * L * H * G * x.splits * (d + 4) * 4 if x.splits > 1 else 0)
        assert x.rows in ((128, 256) if x.many else (16, 32)) and x.splits >= 1
        assert x.waves == x.rows // 32 if x.many else x.waves in (4, 8, 12, 16)
        assert not (x.many and (dtype == cq.CQSA_F32 or L * G <= 64))


def test_refused_and_empty():
    lib, out = cq.lib(), cq.cqsa_attend_launch(7, 7, 7, 7)
    refused(lib.cqsa_cache_attend_launch(cache(), batch(), view(), None), "out is NULL")
    refused(lib.cqsa_cache_attend_launch(cache(), batch(B=5), view(), out), "B differs")
    assert (out.many, out.rows, out.waves, out.splits) == (0, 0, 0, 0)
    x = launch(cache(), batch(), view(L=0, data=None))
    assert (x.many, x.rows, x.waves, x.splits) == (0, 0, 0, 0)
    assert launch(cache(), batch(), view(data=PTR)).rows == 16


def test_ragged_batches_are_not_refused_by_rows_that_no_sequence_has():
    """A chunk of 8192 rows beside 1023 single tokens: the grid that max_q asks for has 2^24 work
    groups, more than one dimension of a grid takes."""
    for dtype, most in ((cq.CQSA_BF16, 1 << 20), (cq.CQSA_F32, 1 << 24)):
        c, b = cache(H=8), long_batch(1024, 1 << 14, q_start=PTR, max_q=8192)
        q = view(B=1, L=8192 + 1023, H=32, dtype=dtype)
        x = launch(c, b, q)
        assert x.splits * 1024 * 8 * 8192 * 4 // x.rows == most


@pytest.mark.parametrize("kw", [dict(max_len=(1 << 32) + 300), dict(max_q=(1 << 32) + 1), dict(max_len=1 << 31), dict(max_q=-1)])
def test_bounds_that_their_fields_do_not_hold(kw):
    """The C structure has 32 bits: 2^32 + 300 would be a bound of 300, and tokens past it left out."""
    with pytest.raises(ValueError, match="2\\^31"):
        cq.CacheBatch(None, None, **kw)


@pytest.mark.parametrize("kw", [dict(d=(1 << 32) + 64), dict(d=64, sections=((1 << 32) + 16, 16))])
def test_rotations_that_their_fields_do_not_hold(kw):
    with pytest.raises(ValueError, match="2\\^31"):
        cq.cqsa_rotary_plan(**kw)


def test_caches_that_their_fields_do_not_hold():
    with pytest.raises(ValueError, match="2\\^31"):
        cq.Cache4(1, (1 << 32) + 8, 64)


@pytest.mark.parametrize("dtype,d,rows,length,many", [
    (cq.CQSA_BF16, 32, 70, 1000, 0), (cq.CQSA_BF16, 32, 140, 1000, 0), (cq.CQSA_BF16, 32, 256, 100, 1), (cq.CQSA_BF16, 32, 100, 128, 1),
    (cq.CQSA_BF16, 64, 70, 300, 0), (cq.CQSA_BF16, 64, 128, 300, 1), (cq.CQSA_BF16, 64, 140, 1000, 0), (cq.CQSA_BF16, 64, 256, 1000, 1),
    (cq.CQSA_BF16, 96, 70, 300, 0), (cq.CQSA_BF16, 96, 140, 1000, 1), (cq.CQSA_BF16, 128, 70, 1000, 0), (cq.CQSA_BF16, 128, 70, 300, 1),
    (cq.CQSA_BF16, 160, 100, 1000, 1), (cq.CQSA_BF16, 224, 70, 1000, 1), (cq.CQSA_BF16, 256, 70, 1000, 0), (cq.CQSA_F16, 64, 70, 1000, 0),
    (cq.CQSA_F16, 192, 70, 1000, 0), (cq.CQSA_F16, 224, 140, 300, 0), (cq.CQSA_F16, 224, 128, 1000, 1), (cq.CQSA_F32, 128, 256, 100, 0)])
def test_rows_that_fill_a_work_group_in_part(dtype, d, rows, length, many):
    """64 sequences and 8 key heads fill the GPU unsplit: the kernel for many rows where its work groups are
    full enough for the length, by the times at the rule."""
    x = launch(cache(H=8, d=d), long_batch(64, length), view(B=64, L=rows, H=8, d=d, dtype=dtype))
    assert x.many == many and (x.splits == 1 or not many)


@pytest.mark.parametrize("d,rows,length,many", [(64, 2048, 4096, 1), (96, 2048, 4096, 0), (128, 2048, 4096, 0), (128, 2048, 5120, 1),
                                                (128, 2048, 8192, 1), (192, 1024, 4096, 1), (192, 1024, 2048, 0)])
def test_units_that_a_split_call_needs(d, rows, length, many):
    """One sequence and 8 key heads: 2^17 units of 16 rows by 32 tokens, 5 / 4 of that at d = 96 and 128."""
    assert launch(cache(H=8, d=d), long_batch(1, length), view(B=1, L=rows, H=8, d=d)).many == many
