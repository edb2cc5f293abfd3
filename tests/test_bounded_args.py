"""Refusals of cqsa_cache_weigh, cqsa_cache_evict and cqsa_draft_verify, and their workspaces: all without a
GPU.  Device pointers here are never read: every call ends at its checks."""
import ctypes

import numpy as np
import pytest

import paper_2604_20819_amd as cq
from oracle import bounded as ob
from tests.test_operator_args import PTR, cache, refused, view

FAR = 1 << 34
SPACE = PTR + 4 * FAR


def batch(**kw):
    b = cq.cqsa_cache_batch(PTR + 6 * FAR, 5, PTR + 7 * FAR, None, 2, 5, 300, 0)
    for k, x in kw.items():
        setattr(b, k, x)
    return b


def weights(T=300, B=2, H=4, data=PTR + FAR, **kw):
    w = cq.cqsa_weights(data, B, H, T, H * T, T)
    for k, x in kw.items():
        setattr(w, k, x)
    return w


def unsupported(status, text):
    assert status == -2 and text in cq.lib().cqsa_last_error().decode()


# -------------------------------------------------------------------- weigh
def weigh(c=None, b=None, q=None, lse=PTR + 2 * FAR, counts=None, prior=None, decay=1.0, w=None, causal=1, scale=0.0, space=SPACE,
          size=1 << 40):
    return cq.lib().cqsa_cache_weigh(c or cache(), b or batch(), q or view(H=8), lse, counts, prior, decay,
                                     w or weights(), causal, scale, space, size, None)


def test_weigh_refused():
    refused(weigh(c=cache(d=48)), "multiple of 32")
    refused(weigh(b=batch(max_len=400)), "max_len")
    refused(weigh(b=batch(B=3)), "B differs")
    refused(weigh(q=view(H=6)), "multiple of the cache's")
    refused(weigh(q=view(H=8, d=96)), "d differs")
    refused(weigh(q=view(H=8, data=PTR + 8)), "16-byte aligned")
    refused(weigh(causal=2), "causal")
    refused(weigh(scale=float("nan")), "scale")
    for bad in (-0.1, 1.5, float("nan"), float("inf")):
        refused(weigh(decay=bad), "decay")
    refused(weigh(w=weights(T=299)), "T = 300 or more")
    refused(weigh(w=weights(B=3)), "B and H differ")
    refused(weigh(w=weights(H=8)), "B and H differ")
    refused(weigh(w=weights(data=None)), "W.data is NULL")
    refused(weigh(w=weights(data=PTR + FAR + 2)), "4-byte aligned")
    refused(weigh(w=weights(stride_h=299)), "overlaps itself")
    refused(weigh(w=weights(stride_h=0)), "overlaps itself")
    refused(weigh(w=weights(stride_b=1100)), "overlaps itself")
    refused(weigh(w=weights(stride_b=-1200)), "strides")
    refused(weigh(prior=weights(T=10)), "prior must have T")
    refused(weigh(prior=weights(data=PTR + FAR + 4)), "W overlaps prior")
    refused(weigh(prior=weights(stride_h=600, stride_b=2400)), "W overlaps prior")
    refused(weigh(lse=None), "LSE is NULL")
    refused(weigh(lse=PTR + 2), "4-byte")
    refused(weigh(lse=PTR + FAR + 64), "W overlaps LSE")
    refused(weigh(counts=PTR + FAR), "W overlaps counts")
    refused(weigh(counts=PTR + 1), "4-byte")
    refused(weigh(w=weights(data=PTR)), "W overlaps the cache")
    refused(weigh(b=batch(pages=PTR + FAR + 8)), "W overlaps the pages")
    refused(weigh(b=batch(lengths=PTR + FAR + 9592)), "W overlaps the lengths")
    refused(weigh(q=view(H=8, data=PTR + FAR - 64)), "W overlaps Q")
    refused(weigh(q=view(B=1, L=6, H=8, data=PTR + 3 * FAR), b=batch(q_start=PTR + FAR, max_q=6)), "W overlaps q_start")
    refused(weigh(b=batch(lengths=None)), "lengths is NULL")
    refused(weigh(b=batch(pages=None)), "pages is NULL")
    assert cq.lib().cqsa_cache_weigh(cache(), batch(), view(H=8), PTR, None, None, 1.0, None, 1, 0.0, None, 0, None) == -1
    # axes of one element have any stride
    assert weigh(b=batch(B=1, lengths=None), q=view(B=1, H=8), w=weights(B=1, stride_b=0)) == -1
    assert "lengths is NULL" in cq.lib().cqsa_last_error().decode()
    # nothing to do
    assert weigh(b=batch(B=0, lengths=None), q=view(B=0, H=8, data=None), w=weights(B=0, data=None)) == 0
    assert weigh(b=batch(max_len=0, lengths=None), w=weights(T=0, data=None)) == 0


def test_weigh_without_rows_and_a_negative_bound_refused():
    """n_b would be max_q, below 0, and prior be read behind its tokens."""
    n = ctypes.c_uint64()
    none = view(B=1, L=0, H=8, data=None)
    b = batch(q_start=PTR + 5 * FAR, max_q=-5, lengths=None)  # no lengths: the call ends at its checks in any case
    refused(weigh(b=b, q=none, prior=weights()), "max_q")
    refused(cq.lib().cqsa_cache_weigh_workspace(cache(), b, none, n), "max_q")
    b.max_q = 0
    refused(weigh(b=b, q=none, prior=weights()), "lengths is NULL")
    assert cq.lib().cqsa_cache_weigh_workspace(cache(), b, none, n) == 0 and n.value == 0


def test_weigh_workspace():
    n = ctypes.c_uint64(7)
    assert cq.lib().cqsa_cache_weigh_workspace(cache(), batch(), view(H=8), n) == 0
    assert cq.lib().cqsa_cache_weigh_workspace(cache(), batch(), view(H=8), None) == -1
    refused(cq.lib().cqsa_cache_weigh_workspace(cache(H=3), batch(), view(H=8), n), "multiple of the cache's")
    for B, L, Hq, max_len in ((1, 1, 8, 300), (1, 2048, 16, 300), (1, 4096, 8, 32), (64, 300, 8, 300)):
        q, b = view(B=B, L=L, H=Hq), batch(B=B, max_len=max_len)
        assert cq.lib().cqsa_cache_weigh_workspace(cache(), b, q, n) == 0
        if n.value:
            w = weights(B=B)
            refused(weigh(b=b, q=q, w=w, space=None), "workspace")
            refused(weigh(b=b, q=q, w=w, size=n.value - 1), "workspace")
            refused(weigh(b=b, q=q, w=w, space=SPACE + 4), "workspace")
            refused(weigh(b=b, q=q, w=w, space=w.data + 16), "overlaps")
        assert n.value < 1 << 30


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("d", [32, 128, 256])
def test_weigh_workspace_of_long_bounds(d, dtype):
    """The parts of a split call are bounded, however long a bound the caller gives for the lengths."""
    n = ctypes.c_uint64()
    for B, L, Hq, max_len in ((1, 65536, 64, 1 << 24), (7, 4096, 64, 1 << 20), (1000, 4096, 64, 1 << 20), (64, 4096, 128, 4096),
                              (2, 8192, 32, 8192)):
        c, q = cache(d=d, n_pages=1 << 20), view(B=B, L=L, H=Hq, d=d, dtype=dtype)
        b = batch(B=B, max_len=max_len, max_pages=max_len, pages_stride=max_len)
        assert cq.lib().cqsa_cache_weigh_workspace(c, b, q, n) == 0, cq.lib().cqsa_last_error()
        assert n.value <= 1 << 27


def test_missing_tensors_are_named():
    """The binding's checks of tensors that a call cannot do without; None is refused as other wrong ones are."""
    import torch
    q = torch.zeros(2, 3, 4, 64)
    with pytest.raises(ValueError, match="LSE must be"):
        cq._lse(None, q, q.device)
    with pytest.raises(ValueError, match="W must be"):
        cq._weights(None, "W", q.device)
    with pytest.raises(ValueError, match="target must be"):
        cq._probs(None, "target", q.device)


# -------------------------------------------------------------------- evict
def opts(budget=100, first=0, recent=0):
    return cq.cqsa_evict_opts(budget, first, recent)


def tables(**kw):
    b = cq.cqsa_cache_batch(PTR + 3 * FAR, 5, None, None, 2, 5, 0, 0)
    for k, x in kw.items():
        setattr(b, k, x)
    return b


def evict(c=None, b=None, w=None, o=None, to=None, w_to=None, kept=None, new=PTR + 2 * FAR, space=SPACE, size=1 << 40):
    return cq.lib().cqsa_cache_evict(c or cache(), b or batch(), w or weights(), o or opts(), to, w_to, kept, new, space, size,
                                     None)


def test_evict_refused():
    refused(cq.lib().cqsa_cache_evict(cache(), batch(), weights(), None, None, None, None, PTR, None, 0, None), "opts is NULL")
    for bad in (0, -5):
        refused(evict(o=opts(bad)), "budget")
    for bad in (opts(10, -1, 0), opts(10, 0, -1), opts(10, 5, 6), opts(10, 2 ** 31 - 1, 2 ** 31 - 1)):
        refused(evict(o=bad), "first and recent")
    refused(evict(c=cache(page_size=48)), "page_size")
    refused(evict(b=batch(max_len=400)), "max_len")
    refused(evict(w=weights(T=200)), "T = 300 or more")
    refused(evict(w=weights(stride_h=10)), "overlaps itself")  # in place it is written
    refused(evict(w_to=weights()), "W_to must be NULL")
    refused(evict(to=tables(), w_to=weights(T=99, data=PTR + 5 * FAR)), "W_to must have T = 100")
    refused(evict(to=tables(), w_to=weights(T=100, data=PTR + FAR + 16)), "W_to overlaps W")
    refused(evict(to=tables(), w=weights(stride_h=10, stride_b=0), w_to=weights(T=100, stride_h=99)), "overlaps itself")
    refused(evict(to=tables(B=3)), "to.B")
    refused(evict(to=tables(max_pages=1)), "pages for")
    refused(evict(to=tables(pages_stride=4)), "to.pages_stride")
    refused(evict(to=tables(pages=None)), "to.pages")
    refused(evict(to=tables(pages=PTR + 2)), "to.pages")
    refused(evict(new=None), "new_lengths")
    refused(evict(new=PTR + 2), "new_lengths")
    refused(evict(new=PTR + FAR + 400), "new_lengths overlaps W")
    refused(evict(new=PTR), "new_lengths overlaps the cache")
    refused(evict(kept=PTR + 2), "kept")
    refused(evict(kept=PTR + FAR + 1200), "kept overlaps W")
    refused(evict(kept=PTR + 2 * FAR), "kept overlaps new_lengths")
    refused(evict(b=batch(lengths=PTR + 2 * FAR - 4)), "new_lengths overlaps the lengths")
    refused(evict(kept=PTR + 6 * FAR), "kept overlaps the pages")
    refused(evict(to=tables(), new=PTR + 3 * FAR + 36), "new_lengths overlaps to's pages")
    refused(evict(space=None), "workspace")
    refused(evict(space=SPACE + 8), "workspace")
    refused(evict(space=PTR), "overlaps the workspace")
    refused(evict(b=batch(lengths=None)), "lengths is NULL")
    unsupported(evict(c=cache(H=65536), b=batch(B=129), w=weights(B=129, H=65536)), "one launch")
    assert evict(b=batch(B=0, lengths=None), w=weights(B=0, data=None), new=None) == 0


def test_evict_workspace():
    n, m = ctypes.c_uint64(), ctypes.c_uint64()
    f = cq.lib().cqsa_cache_evict_workspace
    assert f(cache(), batch(), 100, 0, n) == 0 and f(cache(), batch(), 100, 1, m) == 0
    # in place: 4 tiles of each of 8 heads, and their weights, pass through it
    assert m.value - n.value == 8 * 4 * 34 * 64 + 8 * 100 * 4
    refused(evict(size=m.value - 1), "the call needs")
    refused(evict(to=tables(), size=n.value - 1), "the call needs")
    refused(f(cache(), batch(), 0, 0, n), "budget")
    refused(f(cache(), batch(), 1, 2, n), "in_place")
    assert f(cache(), batch(), 1, 0, None) == -1
    assert f(cache(), batch(B=0), 1, 0, n) == 0 and n.value == 0


# ------------------------------------------------------------------- verify
def probs(N, B=2, V=50, data=PTR, dtype=cq.CQSA_BF16, **kw):
    p = cq.cqsa_probs(data, dtype, B, N, V, N * V, V)
    for k, x in kw.items():
        setattr(p, k, x)
    return p


def verify(p=None, q=0, tokens=PTR + FAR, counts=None, u=PTR + 2 * FAR, out=PTR + 3 * FAR, n_out=PTR + 4 * FAR, lengths=None,
           new=None, space=PTR + 6 * FAR, size=1 << 30):
    q = probs(3, data=PTR + 5 * FAR) if q == 0 else q
    return cq.lib().cqsa_draft_verify(p or probs(4), q, tokens, counts, u, out, n_out, lengths, new, space, size, None)


def test_verify_refused():
    f = cq.lib().cqsa_draft_verify
    refused(f(None, None, PTR, None, PTR, PTR, PTR, None, None, None, 0, None), "target is NULL")
    refused(verify(p=probs(1)), "K in [1, 64]")
    refused(verify(p=probs(66)), "K in [1, 64]")
    refused(verify(p=probs(4, V=0)), "V must be")
    refused(verify(p=probs(4, V=2 ** 24 + 1)), "V must be")
    refused(verify(p=probs(4, B=-1)), "B must be")
    refused(verify(p=probs(4, B=2 ** 20 + 1)), "B must be")
    refused(verify(p=probs(4, dtype=5)), "dtype")
    refused(verify(p=probs(4, stride_n=-50)), "strides")
    refused(verify(p=probs(4, data=None)), "target.data")
    refused(verify(p=probs(4, data=PTR + 1)), "target.data")
    refused(verify(p=probs(4, dtype=cq.CQSA_F32, data=PTR + 2), q=None), "target.data")
    refused(verify(q=probs(4)), "draft must be")
    refused(verify(q=probs(3, V=49)), "draft must be")
    refused(verify(q=probs(3, B=1)), "draft must be")
    refused(verify(q=probs(3, dtype=cq.CQSA_F16)), "draft must be")
    refused(verify(q=probs(3, data=None)), "draft.data")
    for name in ("tokens", "u", "out", "n_out"):
        refused(verify(**{name: None}), f"{name} is NULL")
        refused(verify(**{name: PTR + 7 * FAR + 2}), "4-byte")
    refused(verify(counts=PTR + 2), "4-byte")
    refused(verify(lengths=PTR + 7 * FAR), "or neither")
    refused(verify(new=PTR + 7 * FAR), "or neither")
    refused(verify(lengths=PTR + 7 * FAR, new=PTR + 7 * FAR + 4), "new_lengths overlaps lengths")
    refused(verify(out=PTR + FAR), "out overlaps tokens")
    refused(verify(out=PTR + 2 * FAR - 8), "out overlaps u")
    refused(verify(n_out=PTR + 64), "n_out overlaps target")
    refused(verify(n_out=PTR + 5 * FAR), "n_out overlaps draft")
    refused(verify(n_out=PTR + 3 * FAR + 8), "out overlaps n_out")
    refused(verify(counts=PTR + 4 * FAR + 4), "n_out overlaps counts")
    refused(verify(lengths=PTR + 3 * FAR, new=PTR + 3 * FAR), "overlaps")
    assert verify(p=probs(4, B=0, data=None), q=None, tokens=None, u=None, out=None, n_out=None) == 0


def test_verify_workspace():
    n = ctypes.c_uint64()
    f = cq.lib().cqsa_draft_verify_workspace
    refused(f(probs(1), n), "K in [1, 64]")
    assert f(probs(4), None) == -1
    for B in (1, 3, 70, 300):
        for V in (1, 1000, 131072):
            assert f(probs(4, B=B, V=V), n) == 0 and n.value < 1 << 26
            if n.value:
                p = probs(4, B=B, V=V)
                far = 1 << 36
                at = dict(tokens=PTR + far, u=PTR + 2 * far, out=PTR + 3 * far, n_out=PTR + 4 * far)
                refused(verify(p=p, q=None, space=None, **at), "workspace")
                refused(verify(p=p, q=None, space=PTR + 5 * far, size=n.value - 1, **at), "workspace")
                refused(verify(p=p, q=None, space=PTR + 5 * far + 8, **at), "workspace")
                refused(verify(p=p, q=None, space=PTR + 3 * far, **at), "overlaps")


# ------------------------------------------------------------------ oracles
def test_oracle_keep():
    w = np.array([5.0, 1.0, 3.0, 3.0, np.nan, 0.0, -0.0, 2.0])
    yes = np.ones(8, bool)
    assert ob.keep(w, yes, 8, 8, 0, 0) == list(range(8))
    assert ob.keep(w, yes, 8, 2, 0, 0) == [0, 2]
    assert ob.keep(w, yes, 8, 3, 0, 1) == [0, 2, 7]
    assert ob.keep(w, yes, 8, 5, 2, 1) == [0, 1, 2, 3, 7]
    assert ob.keep(w, yes, 8, 6, 0, 0) == [0, 1, 2, 3, 5, 7]  # of equal zeros the earlier
    assert ob.keep(w, yes, 5, 9, 0, 0) == [0, 1, 2, 3, 4]
    there = yes.copy()
    there[[0, 7]] = False
    assert ob.keep(w, there, 8, 3, 1, 1) == [1, 2, 3]


def test_oracle_verify():
    p = np.array([[0.5, 0.5, 0.0], [0.2, 0.3, 0.5]])
    q = np.array([[0.0, 0.6, 0.4]])
    assert ob.verify(p, q, [1], 1, np.array([0.8, 0.1]))[:3] == (pytest.approx([1, 0]), 2, None)
    assert ob.verify(p, q, [1], 1, np.array([0.9, 0.99]), 10)[1:3] == (1, 9)
    assert ob.verify(p, q, [2], 1, np.array([0.0, 0.99]))[0].tolist() == [0, -1]
    assert ob.verify(p, None, [0], 1, np.array([0.6, 0.0]))[0].tolist() == [1, -1]
    assert ob.verify(p, None, [0], 0, np.array([0.0, 0.5]))[0].tolist() == [1, -1]


def test_oracle_weigh():
    g = np.random.Generator(np.random.PCG64(1))
    q, k = g.standard_normal((3, 4, 32)), g.standard_normal((9, 2, 32))
    x = np.einsum("ihd,thd->iht", q, np.repeat(k, 2, 1)) * 0.25
    for i in range(3):
        x[i, :, 7 + i:] = -np.inf
    lse = np.log(np.exp(x).sum(-1))
    W, _ = ob.weigh(q, k, lse, np.ones(9, bool), 9, 3, True, 0.25, None, 1.0)
    assert W.sum(-1) == pytest.approx(6.0)
    there = np.ones(9, bool)
    there[4] = False
    for causal in (True, False):
        for count in (0, 2, 3):
            a = ob.weigh(q, k, lse, there, 9, count, causal, 0.25, np.ones((2, 9)), 0.5)
            b = ob.weigh_rows(q, k, lse, there, 9, count, causal, 0.25, np.ones((2, 9)), 0.5)
            assert a[0] == pytest.approx(b[0], abs=1e-12) and a[1] == pytest.approx(b[1], abs=1e-12)
    W, _ = ob.weigh(q, k, lse, np.ones(9, bool), 9, 1, True, 0.25, np.ones((2, 9)), 0.5)
    assert W.sum(-1) == pytest.approx(2.0 + 3.0) and (W[:, 7:] == 0).all()
