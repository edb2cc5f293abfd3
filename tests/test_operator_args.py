"""Refusals of the rotary and cache entry points, the plan's table and the format's sizes:
all without a GPU.  Device pointers here are never read: every call ends at its checks."""
import ctypes

import numpy as np
import pytest

import paper_2604_20819_amd as cq
from oracle import cache4 as o4
from oracle import rotary as orot

PTR = 1 << 20  # an aligned address that no call reaches


def view(B=2, L=3, H=4, d=64, dtype=cq.CQSA_BF16, data=PTR, **kw):
    v = cq.cqsa_view(data, dtype, B, L, H, d, L * H * d, H * d, d)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


def cache(**kw):
    c = cq.cqsa_cache(PTR, 10, 64, 4, 64)
    for k, x in kw.items():
        setattr(c, k, x)
    return c


def batch(**kw):
    b = cq.cqsa_cache_batch(PTR, 5, PTR, None, 2, 5, 300, 0)
    for k, x in kw.items():
        setattr(b, k, x)
    return b


def refused(status, text):
    assert status == -1, status
    assert text in cq.lib().cqsa_last_error().decode(), cq.lib().cqsa_last_error()


# ------------------------------------------------------------------- rotary
@pytest.mark.parametrize("kw,text", [
    (dict(d=48), "multiple of 32"), (dict(d=288), "multiple of 32"), (dict(d=0), "multiple of 32"),
    (dict(sections=(16, 0)), "1 pair"), (dict(sections=(16, -8)), "1 pair"),
    (dict(sections=(4, 5)), "multiple of 8"), (dict(sections=(32, 8)), "d / 2"),
    (dict(theta=1.0), "theta"), (dict(theta=float("nan")), "theta"), (dict(theta=float("inf")), "theta"),
    (dict(sections=(16, 16), pos_scale=(1.0, 0.0)), "pos_scale"),
    (dict(sections=(16, 16), pos_scale=(float("nan"), 1.0)), "pos_scale")])
def test_rotary_plans_refused(kw, text):
    with pytest.raises(cq.CqsaError) as e:
        cq.cqsa_rotary_plan(**{"d": 64, **kw})
    assert e.value.status == -1 and text in str(e.value)


def test_rotary_plan_options_refused():
    h = ctypes.c_void_p()
    for name, bad in (("pairs", 2), ("spectrum", -1), ("dealt", 2), ("n_axes", 0), ("n_axes", 5)):
        o = cq.cqsa_rotary_opts()
        cq.lib().cqsa_rotary_opts_default(o, 64)
        setattr(o, name, bad)
        assert cq.lib().cqsa_rotary_plan(o, h) == -1 and not h.value
    assert cq.lib().cqsa_rotary_plan(None, h) == -1
    assert cq.lib().cqsa_rotary_plan(o, None) == -1
    with pytest.raises(ValueError):
        cq.cqsa_rotary_plan(64, (1, 1, 1, 1, 4))
    cq.lib().cqsa_rotary_destroy(None)


def test_rotary_calls_refused():
    plan = cq.cqsa_rotary_plan(64, (16, 16)).handle
    keep = cq.cqsa_rotary_plan(64, (16, 16))
    plan = keep.handle

    def call(x, y, n=1, inverse=0, p=plan, pos=PTR):
        a = (cq.cqsa_view * 2)(*(list(x) * 2)[:2])
        b = (cq.cqsa_view * 2)(*(list(y) * 2)[:2])
        return cq.lib().cqsa_rotary(p, pos, a, b, n, inverse, None)

    far = dict(data=PTR + (1 << 30))
    ok, out = view(), view(**far)
    refused(call([ok], [out], p=None), "plan is NULL")
    refused(call([ok], [out], n=0), "n must be")
    refused(call([ok], [out], n=3), "n must be")
    refused(call([ok], [out], inverse=2), "inverse")
    refused(call([ok], [out], pos=None), "pos is NULL")
    refused(call([ok], [out], pos=PTR + 2), "4-byte")
    refused(call([view(d=96)], [out]), "d differs")
    refused(call([view(dtype=7)], [out]), "unknown dtype")
    refused(call([view(data=None)], [out]), "NULL")
    refused(call([view(data=PTR + 8)], [out]), "16-byte aligned")
    refused(call([view(stride_l=4 * 64 + 4)], [out]), "strides")
    refused(call([view(stride_h=-64)], [out]), "strides")
    refused(call([view(B=-1)], [out]), "extent")
    refused(call([ok], [view(L=4, **far)]), "differs from x")
    refused(call([ok], [view(dtype=cq.CQSA_F16, **far)]), "differs from x")
    refused(call([ok], [view(stride_h=0, **far)]), "overlaps itself")
    refused(call([ok], [view(stride_l=64, **far)]), "overlaps itself")
    refused(call([ok], [view(data=PTR + 16)]), "overlaps x")
    refused(call([ok, view(L=5)], [out, view(L=5, **far)], n=2), "share B, L")
    refused(call([ok, view(dtype=cq.CQSA_F16)], [out, view(dtype=cq.CQSA_F16, **far)], n=2), "share B, L")
    refused(call([ok, ok], [ok, ok], n=2), "one tensor")
    refused(call([ok, view(data=PTR + (1 << 31))], [out, out], n=2), "one tensor")
    assert call([view(B=0, data=None)], [view(B=0, data=None)]) == 0  # nothing to do


def test_rotary_table_by_the_python_binding():
    """The plan is made for every allowed shape of axes."""
    for sections in ((8,), (128,), (1, 1, 1, 125), (40, 40, 48)):
        for spectrum in ("shared", "per_axis"):
            for dealt in (False, True):
                cq.cqsa_rotary_plan(256, sections, spectrum=spectrum, dealt=dealt)
    assert orot.axes_of((1, 3, 2), True) == [(0, 0), (1, 0), (2, 0), (1, 1), (2, 1), (1, 2)]


# -------------------------------------------------------------------- cache
def test_page_bytes():
    for page in (32, 64, 128, 256):
        for H, d in ((1, 32), (8, 128), (3, 224)):
            assert cq.cqsa_cache_page_bytes(page, H, d) == o4.page_bytes(page, H, d)
    for bad in ((48, 1, 64), (0, 1, 64), (512, 1, 64), (64, 0, 64), (64, 1, 48), (64, 1, 288), (64, 65537, 64)):
        assert cq.cqsa_cache_page_bytes(*bad) == 0


def calls():
    far = dict(data=PTR + (1 << 32))
    lib = cq.lib()

    def move(f):
        return lambda c, b, t: f(c, b, t, view_like(t, **far), None)

    def attend(c, b, t):
        return lib.cqsa_cache_attend(c, b, t, view_like(t, **far), PTR, 1, 0.0, PTR, 1 << 40, None)

    return {"write": move(lib.cqsa_cache_write), "read": move(lib.cqsa_cache_read), "attend": attend}


def view_like(t, **kw):
    v = cq.cqsa_view.from_buffer_copy(t)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


@pytest.mark.parametrize("name", ["write", "read", "attend"])
def test_cache_calls_refused(name):
    call = calls()[name]
    t = view()
    refused(call(None, batch(), t), "cache is NULL")
    refused(call(cache(), None, t), "batch is NULL")
    refused(call(cache(page_size=48), batch(), t), "page_size")
    refused(call(cache(page_size=512), batch(), t), "page_size")
    refused(call(cache(d=80), batch(), view(d=80)), "multiple of 32")
    refused(call(cache(H=0), batch(), t), "H must be")
    refused(call(cache(n_pages=-1), batch(), t), "n_pages")
    refused(call(cache(data=None), batch(), t), "data is NULL")
    refused(call(cache(data=PTR + 32), batch(), t), "64-byte")
    refused(call(cache(), batch(B=-1), t), "batch.B")
    refused(call(cache(), batch(B=3), t), "B differs")
    refused(call(cache(), batch(pages_stride=4), t), "pages_stride")
    refused(call(cache(), batch(max_pages=-1), t), "pages_stride")
    refused(call(cache(), batch(max_len=321), t), "max_len")
    refused(call(cache(), batch(max_len=-1), t), "max_len")
    refused(call(cache(), batch(pages=None), t), "pages is NULL")
    refused(call(cache(), batch(lengths=None), t), "lengths is NULL")
    refused(call(cache(), batch(lengths=PTR + 1), t), "4-byte")
    refused(call(cache(), batch(q_start=PTR, max_q=1), t), "B = 1")
    refused(call(cache(), batch(q_start=PTR, max_q=0), view(B=1)), "max_q")
    refused(call(cache(), batch(q_start=PTR, max_q=4), view(B=1)), "max_q")
    refused(call(cache(), batch(), view(d=96)), "d differs")
    refused(call(cache(), batch(), view(data=PTR + 4)), "16-byte")
    refused(call(cache(), batch(), view(stride_l=260)), "strides")
    refused(call(cache(), batch(), view(H=6)), "heads")
    assert call(cache(), batch(B=0), view(B=0, data=None)) == 0
    assert call(cache(), batch(), view(L=0, data=None)) == 0


def test_more_of_attend_refused():
    lib, far = cq.lib(), dict(data=PTR + (1 << 32))

    def call(q=view(), o=view(**far), causal=1, scale=0.0, lse=PTR):
        return lib.cqsa_cache_attend(cache(), batch(), q, o, lse, causal, scale, PTR, 1 << 40, None)

    refused(call(causal=2), "causal")
    refused(call(scale=float("nan")), "scale")
    refused(call(scale=float("inf")), "scale")
    refused(call(scale=3e38), "scale")  # infinite as a factor of powers of two
    refused(call(o=view(stride_h=3 * 64, stride_l=64)), "without being Q")
    refused(call(lse=PTR + 2), "LSE")
    refused(call(o=view(L=4, **far)), "O differs")
    refused(call(o=view(dtype=cq.CQSA_F32, **far)), "O differs")
    refused(call(o=view(stride_h=0, **far)), "overlaps itself")
    refused(call(q=view(H=2)), "heads")
    refused(call(q=None), "Q is NULL")
    refused(lib.cqsa_cache_attend_workspace(cache(), batch(), view(), None), "bytes is NULL")
    n = ctypes.c_uint64(7)
    refused(lib.cqsa_cache_attend_workspace(cache(), batch(B=5), view(), n), "B differs")
    assert n.value == 0


def test_calls_too_large_for_a_launch():
    lib, far = cq.lib(), dict(data=PTR + (1 << 40))
    n = ctypes.c_uint64()

    def unsupported(status):
        assert status == -2 and "launch" in lib.cqsa_last_error().decode()

    B = 1 << 20
    many = view(B=B, L=1, H=16, stride_b=0)
    c, b = cache(H=16), batch(B=B, max_pages=5, pages_stride=5)
    for f in (lib.cqsa_cache_write, lib.cqsa_cache_read):
        out = view(B=B, L=1, H=16, stride_b=16 * 64, **far)
        unsupported(f(c, b, out, out, None))
    unsupported(lib.cqsa_cache_attend_workspace(c, b, many, n))
    long = view(B=1, L=1 << 30, H=4, stride_b=0, stride_l=0)
    unsupported(lib.cqsa_cache_attend_workspace(cache(H=1), batch(B=1), long, n))
    unsupported(lib.cqsa_cache_attend_workspace(cache(), batch(B=8), view(B=8, L=1 << 29, stride_b=0, stride_l=0), n))
    keep = cq.cqsa_rotary_plan(64)
    wide = view(B=1, L=1, H=(1 << 20) + 1)
    assert lib.cqsa_rotary(keep.handle, PTR, wide, view(B=1, L=1, H=(1 << 20) + 1, **far), 1, 0, None) == -2


def test_workspace_by_the_sizes_alone():
    """None for short contexts; splits x rows x (d + 4) floats for long ones, also where Q's data is not there."""
    lib, n = cq.lib(), ctypes.c_uint64(7)
    q = view(L=1)
    assert lib.cqsa_cache_attend_workspace(cache(), batch(), q, n) == 0 and n.value == 0
    b = batch(max_pages=1 << 14, pages_stride=1 << 14, max_len=1 << 20)
    assert lib.cqsa_cache_attend_workspace(cache(), b, q, n) == 0 and n.value > 0
    assert n.value % (2 * 4 * (64 + 4) * 4) == 0
    # too small, missing and misaligned ones are refused
    for space, size, text in ((None, 0, "workspace"), (PTR, n.value - 1, "workspace"), (PTR + 8, n.value, "16-byte")):
        refused(lib.cqsa_cache_attend(cache(), b, q, view(L=1, data=PTR + (1 << 32)), None, 1, 0.0, space, size, None), text)


def test_workspace_of_many_rows():
    """One key head's rows are split to fill the GPU, rows that fill it by themselves are not split."""
    lib, n = cq.lib(), ctypes.c_uint64(7)
    b = batch(B=1, max_pages=1 << 14, pages_stride=1 << 14, max_len=1 << 20)
    assert lib.cqsa_cache_attend_workspace(cache(H=1), b, view(B=1, L=64), n) == 0
    splits, rest = divmod(n.value, 64 * 4 * (64 + 4) * 4)
    assert rest == 0 and 128 < splits <= 256
    b = batch(B=64, max_len=128)
    assert lib.cqsa_cache_attend_workspace(cache(H=4), b, view(B=64, L=128, H=16), n) == 0 and n.value == 0


def test_batches_and_caches_are_made_once():
    """Their descriptors hold addresses, which an assignment would leave behind."""
    for kind, names in ((cq.CacheBatch, ("lengths", "pages", "max_len")), (cq.Cache4, ("data", "n_pages"))):
        x = object.__new__(kind)
        for name in names:
            with pytest.raises(AttributeError, match="made once"):
                setattr(x, name, None)


def test_write_and_read_views_refused():
    lib = cq.lib()
    for f in (lib.cqsa_cache_write, lib.cqsa_cache_read):
        refused(f(cache(), batch(), view(), view(L=4), None), "K and V differ")
        refused(f(cache(), batch(), view(), view(dtype=cq.CQSA_F32), None), "K and V differ")
    refused(lib.cqsa_cache_read(cache(), batch(), view(), view(stride_h=0), None), "overlaps itself")
    refused(lib.cqsa_cache_read(cache(), batch(), view(), view(), None), "one tensor")


# ---------------------------------------------------- the oracle, by itself
def test_oracle_rounds_to_the_nearest_level():
    """The oracle's codes are the nearest of the sixteen levels (ties to even), and a block's
    power keeps its largest within a factor 7 / 6 of the last level."""
    g = np.random.Generator(np.random.PCG64(1))
    x = g.standard_normal((50, 64)) * 10.0 ** g.integers(-6, 6, (50, 1))
    code, byte = o4.quantise(x)
    v = o4.values(code, byte)
    scale = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=-1)
    levels = np.concatenate([o4.LEVELS, -o4.LEVELS])
    best = np.abs(x[..., None] / scale[..., None] - levels).min(-1)
    assert np.array_equal(np.abs(x / scale - v / scale), best)
    top = np.abs(x.reshape(50, 2, 32)).max(-1) / 2.0 ** (byte.astype(float) - 127)
    assert (top < 7).all() and (top >= 3.5).all()


def test_oracle_places_are_a_permutation():
    for page, H, d in ((32, 1, 32), (64, 3, 96), (256, 2, 128)):
        seen = np.zeros(o4.page_bytes(page, H, d), int)
        for h in range(H):
            for t in range(page):
                for p in o4.places(page, d, h, t):
                    seen[p] += 1
        assert (seen == 1).all()
