"""Stream-CQSA hot path for AMD MI355X: thin ctypes binding of libcqsa.so.

The binding only marshals arguments: every step of planning and compute runs
in the native library (C++ planner, HIP kernels for gfx950).  PyTorch is used
for device memory and streams.  The binding fails loudly when the library has
not been built (``python -m paper_2604_20819_amd.build``); there is no CPU or
eager fallback.

Names follow include/cqsa.h: ``cqsa_plan``, ``cqsa_forward``,
``cqsa_backward``, ``cqsa_set_timing``, ``cqsa_last_stats``,
``cqsa_rotary``, ``cqsa_cache_write``, ``cqsa_cache_attend``, ``cqsa_cache_weigh``,
``cqsa_cache_evict``, ``cqsa_draft_verify`` ...
"""
import ctypes
import os
import struct

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libcqsa.so")

CQSA_F32, CQSA_F16, CQSA_BF16 = 0, 1, 2
CQSA_MEM_HOST, CQSA_MEM_DEVICE = 0, 1
STATUS = {0: "CQSA_OK", -1: "CQSA_ERR_INVALID_ARG", -2: "CQSA_ERR_UNSUPPORTED",
          -3: "CQSA_ERR_BUDGET", -4: "CQSA_ERR_DEVICE_OOM", -5: "CQSA_ERR_HIP",
          -6: "CQSA_ERR_INTERNAL"}


class CqsaError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class cqsa_tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("where", ctypes.c_int),
                ("B", ctypes.c_int64), ("L", ctypes.c_int64), ("H", ctypes.c_int64),
                ("d", ctypes.c_int64)]


class cqsa_interest_set(ctypes.Structure):
    _fields_ = [("c", ctypes.c_int32), ("l", ctypes.c_int32), ("interest", ctypes.c_int32 * 16)]


class cqsa_plan_opts(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("dtype", ctypes.c_int), ("c", ctypes.c_int32),
                ("l", ctypes.c_int32), ("interest", ctypes.c_int32 * 16),
                ("depth", ctypes.c_int32), ("min_depth", ctypes.c_int32),
                ("max_depth", ctypes.c_int32), ("n_slots", ctypes.c_int32),
                ("inputs_on_device", ctypes.c_int32), ("acc_on_device", ctypes.c_int32),
                ("with_backward", ctypes.c_int32), ("tasks_per_slot", ctypes.c_int32),
                ("n_level_sets", ctypes.c_int32), ("level_sets", cqsa_interest_set * 4),
                ("read_in_place", ctypes.c_int32),
                ("out16", ctypes.c_int32), ("bwd_tasks_per_launch", ctypes.c_int32)]


class cqsa_run(ctypes.Structure):
    _fields_ = [("global_start", ctypes.c_int64), ("length", ctypes.c_int64),
                ("bits", ctypes.c_uint32)]


class cqsa_task(ctypes.Structure):
    _fields_ = [("index", ctypes.c_int64), ("depth", ctypes.c_int32),
                ("quorum", ctypes.POINTER(ctypes.c_int32)), ("L_local", ctypes.c_int64),
                ("n_runs", ctypes.c_int32), ("runs", ctypes.POINTER(cqsa_run)),
                ("n_blocks", ctypes.c_int64), ("block_or", ctypes.POINTER(ctypes.c_uint32)),
                ("block_and", ctypes.POINTER(ctypes.c_uint32))]


class cqsa_run_stats(ctypes.Structure):
    _fields_ = [("depth", ctypes.c_int32), ("num_tasks", ctypes.c_int64),
                ("modelled_device_bytes", ctypes.c_uint64), ("workspace_bytes", ctypes.c_uint64),
                ("h2d_bytes", ctypes.c_uint64), ("d2h_bytes", ctypes.c_uint64),
                ("d2d_bytes", ctypes.c_uint64), ("inner_launches", ctypes.c_int64),
                ("ms_wall", ctypes.c_double), ("ms_stage", ctypes.c_double),
                ("ms_inner", ctypes.c_double), ("ms_merge", ctypes.c_double),
                ("ms_finalize", ctypes.c_double), ("ms_d2h", ctypes.c_double),
                ("tiles_full", ctypes.c_int64), ("tiles_clear", ctypes.c_int64),
                ("tiles_mixed", ctypes.c_int64), ("merge_launches", ctypes.c_int64),
                ("ms_inner_busy", ctypes.c_double), ("guard_steps", ctypes.c_int64),
                ("resident_tasks", ctypes.c_int64), ("kernel_tiles_masked", ctypes.c_int64),
                ("kernel_tiles_clear", ctypes.c_int64), ("kernel_tiles_mixed", ctypes.c_int64),
                ("kernel_kv_tiles_masked", ctypes.c_int64), ("kernel_kv_tiles_clear", ctypes.c_int64),
                ("kernel_kv_tiles_mixed", ctypes.c_int64)]


class cqsa_view(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("B", ctypes.c_int64),
                ("L", ctypes.c_int64), ("H", ctypes.c_int64), ("d", ctypes.c_int64),
                ("stride_b", ctypes.c_int64), ("stride_l", ctypes.c_int64),
                ("stride_h", ctypes.c_int64)]


class cqsa_rotary_opts(ctypes.Structure):
    _fields_ = [("d", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("sections", ctypes.c_int32 * 4),
                ("pairs", ctypes.c_int32), ("spectrum", ctypes.c_int32), ("dealt", ctypes.c_int32),
                ("theta", ctypes.c_double), ("pos_scale", ctypes.c_double * 4)]


class cqsa_cache(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32)]


class cqsa_cache_batch(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("pages_stride", ctypes.c_int64),
                ("lengths", ctypes.c_void_p), ("q_start", ctypes.c_void_p),
                ("B", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("max_len", ctypes.c_int32),
                ("max_q", ctypes.c_int32)]


class cqsa_attend_launch(ctypes.Structure):
    _fields_ = [("many", ctypes.c_int32), ("rows", ctypes.c_int32), ("waves", ctypes.c_int32),
                ("splits", ctypes.c_int32)]


class cqsa_weights(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("B", ctypes.c_int64), ("H", ctypes.c_int64), ("T", ctypes.c_int64),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64)]


class cqsa_evict_opts(ctypes.Structure):
    _fields_ = [("budget", ctypes.c_int32), ("first", ctypes.c_int32), ("recent", ctypes.c_int32)]


class cqsa_probs(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("dtype", ctypes.c_int), ("B", ctypes.c_int64), ("N", ctypes.c_int64),
                ("V", ctypes.c_int64), ("stride_b", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


_W, _E, _P = (ctypes.POINTER(x) for x in (cqsa_weights, cqsa_evict_opts, cqsa_probs))
_V, _C, _CB = (ctypes.POINTER(x) for x in (cqsa_view, cqsa_cache, cqsa_cache_batch))

# Every symbol include/cqsa.h declares, with its ctypes signature.
_SIGS = {
    "cqsa_plan_opts_default": (None, [ctypes.POINTER(cqsa_plan_opts)]),
    "cqsa_plan": (ctypes.c_int, [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                 ctypes.c_uint64, ctypes.POINTER(cqsa_plan_opts),
                                 ctypes.POINTER(ctypes.c_void_p)]),
    "cqsa_plan_depth": (ctypes.c_int32, [ctypes.c_void_p]),
    "cqsa_plan_num_tasks": (ctypes.c_int64, [ctypes.c_void_p]),
    "cqsa_plan_get_task": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_int64, ctypes.POINTER(cqsa_task)]),
    "cqsa_plan_modelled_device_bytes": (ctypes.c_uint64, [ctypes.c_void_p]),
    "cqsa_plan_tasks_per_slot": (ctypes.c_int32, [ctypes.c_void_p]),
    "cqsa_plan_bwd_tasks_per_launch": (ctypes.c_int32, [ctypes.c_void_p]),
    "cqsa_plan_acc_on_device": (ctypes.c_int32, [ctypes.c_void_p]),
    "cqsa_plan_reads_in_place": (ctypes.c_int32, [ctypes.c_void_p]),
    "cqsa_plan_tile_census": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                             ctypes.POINTER(ctypes.c_int64),
                                             ctypes.POINTER(ctypes.c_int64)]),
    "cqsa_plan_fwd_tile_decisions": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                                    ctypes.POINTER(ctypes.c_int64),
                                                    ctypes.POINTER(ctypes.c_int64)]),
    "cqsa_bwd_kv_query_tile": (ctypes.c_int32, [ctypes.c_int32]),
    "cqsa_plan_bwd_tile_decisions": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int64),
                                                    ctypes.POINTER(ctypes.c_int64)]),
    "cqsa_plan_destroy": (None, [ctypes.c_void_p]),
    "cqsa_forward": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(cqsa_tensor),
                                    ctypes.POINTER(cqsa_tensor), ctypes.POINTER(cqsa_tensor),
                                    ctypes.POINTER(cqsa_tensor), ctypes.c_void_p, ctypes.c_int,
                                    ctypes.c_float, ctypes.c_void_p]),
    "cqsa_forward_noalloc": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(cqsa_tensor),
                                            ctypes.POINTER(cqsa_tensor), ctypes.POINTER(cqsa_tensor),
                                            ctypes.POINTER(cqsa_tensor), ctypes.c_void_p, ctypes.c_int,
                                            ctypes.c_float, ctypes.c_void_p]),
    "cqsa_backward": (ctypes.c_int, [ctypes.c_void_p, ctypes.POINTER(cqsa_tensor),
                                     ctypes.POINTER(cqsa_tensor), ctypes.POINTER(cqsa_tensor),
                                     ctypes.POINTER(cqsa_tensor), ctypes.c_void_p, ctypes.c_int,
                                     ctypes.POINTER(cqsa_tensor), ctypes.POINTER(cqsa_tensor),
                                     ctypes.POINTER(cqsa_tensor), ctypes.POINTER(cqsa_tensor),
                                     ctypes.c_float, ctypes.c_void_p]),
    "cqsa_rotary_opts_default": (None, [ctypes.POINTER(cqsa_rotary_opts), ctypes.c_int32]),
    "cqsa_rotary_plan": (ctypes.c_int, [ctypes.POINTER(cqsa_rotary_opts),
                                        ctypes.POINTER(ctypes.c_void_p)]),
    "cqsa_rotary_destroy": (None, [ctypes.c_void_p]),
    "cqsa_rotary": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, _V, _V, ctypes.c_int32,
                                   ctypes.c_int32, ctypes.c_void_p]),
    "cqsa_cache_page_bytes": (ctypes.c_uint64, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "cqsa_cache_write": (ctypes.c_int, [_C, _CB, _V, _V, ctypes.c_void_p]),
    "cqsa_cache_read": (ctypes.c_int, [_C, _CB, _V, _V, ctypes.c_void_p]),
    "cqsa_cache_attend": (ctypes.c_int, [_C, _CB, _V, _V, ctypes.c_void_p, ctypes.c_int32,
                                         ctypes.c_float, ctypes.c_void_p, ctypes.c_uint64,
                                         ctypes.c_void_p]),
    "cqsa_cache_attend_workspace": (ctypes.c_int, [_C, _CB, _V, ctypes.POINTER(ctypes.c_uint64)]),
    "cqsa_cache_attend_launch": (ctypes.c_int, [_C, _CB, _V, ctypes.POINTER(cqsa_attend_launch)]),
    "cqsa_cache_weigh": (ctypes.c_int, [_C, _CB, _V, ctypes.c_void_p, ctypes.c_void_p, _W, ctypes.c_float, _W,
                                        ctypes.c_int32, ctypes.c_float, ctypes.c_void_p, ctypes.c_uint64,
                                        ctypes.c_void_p]),
    "cqsa_cache_weigh_workspace": (ctypes.c_int, [_C, _CB, _V, ctypes.POINTER(ctypes.c_uint64)]),
    "cqsa_cache_evict": (ctypes.c_int, [_C, _CB, _W, _E, _CB, _W, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                        ctypes.c_uint64, ctypes.c_void_p]),
    "cqsa_cache_evict_workspace": (ctypes.c_int, [_C, _CB, ctypes.c_int32, ctypes.c_int32,
                                                  ctypes.POINTER(ctypes.c_uint64)]),
    "cqsa_draft_verify": (ctypes.c_int, [_P, _P] + [ctypes.c_void_p] * 8 + [ctypes.c_uint64, ctypes.c_void_p]),
    "cqsa_draft_verify_workspace": (ctypes.c_int, [_P, ctypes.POINTER(ctypes.c_uint64)]),
    "cqsa_set_allocator": (ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]),
    "cqsa_set_timing": (ctypes.c_int, [ctypes.c_int32]),
    "cqsa_set_tile_counting": (ctypes.c_int, [ctypes.c_int32]),
    "cqsa_last_stats": (ctypes.c_int, [ctypes.POINTER(cqsa_run_stats)]),
    "cqsa_release_workspace": (ctypes.c_int, []),
    "cqsa_last_error": (ctypes.c_char_p, []),
}

_lib = None


def lib():
    """The loaded native library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2604_20819_amd.build` (no fallback exists)")
        so = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGS.items():
            fn = getattr(so, name)
            fn.restype = res
            fn.argtypes = args
        _lib = so
    return _lib


def _check(status, what):
    if status != 0:
        msg = lib().cqsa_last_error().decode(errors="replace")
        raise CqsaError(status, f"{what}: {msg}")


def cqsa_plan_opts_default():
    o = cqsa_plan_opts()
    lib().cqsa_plan_opts_default(ctypes.byref(o))
    return o


def make_opts(B=1, dtype="bf16", c=7, interest=(0, 1, 3), depth=-1, min_depth=1, max_depth=4,
              n_slots=2, inputs_on_device=True, acc_on_device=True, with_backward=False,
              tasks_per_slot=0, levels=None, read_in_place=None, out16=False,
              bwd_tasks_per_launch=0):
    """levels: optional list of (c, interest) per depth (the last repeats below).
    acc_on_device=None asks the planner to choose the accumulator residency;
    read_in_place=None lets it choose whether the kernels read the caller's
    tensors in place (True) or gather each task's runs first (False).
    out16=True makes cqsa_forward write O in the input dtype.
    bwd_tasks_per_launch: 0 automatic, n >= 1 backward tasks per launch."""
    o = cqsa_plan_opts_default()
    o.B = B
    o.dtype = {"f32": CQSA_F32, "f16": CQSA_F16, "bf16": CQSA_BF16}[dtype]
    o.c = c
    o.l = len(interest)
    for i in range(16):
        o.interest[i] = interest[i] if i < len(interest) else 0
    o.depth, o.min_depth, o.max_depth, o.n_slots = depth, min_depth, max_depth, n_slots
    o.inputs_on_device = int(bool(inputs_on_device))
    o.acc_on_device = -1 if acc_on_device is None else int(bool(acc_on_device))
    o.with_backward = int(bool(with_backward))
    o.tasks_per_slot = int(tasks_per_slot)
    o.read_in_place = -1 if read_in_place is None else int(bool(read_in_place))
    o.out16 = int(bool(out16))
    o.bwd_tasks_per_launch = int(bwd_tasks_per_launch)
    if levels:
        if len(levels) > 4:
            raise ValueError("at most 4 level sets")
        o.n_level_sets = len(levels)
        for k, (lc, li) in enumerate(levels):
            o.level_sets[k].c = lc
            o.level_sets[k].l = len(li)
            for i in range(16):
                o.level_sets[k].interest[i] = li[i] if i < len(li) else 0
    return o


class Plan:
    """Owner of a cqsa_plan_t*."""

    def __init__(self, handle, opts, L, H, d, causal):
        self.handle = handle
        self.opts = opts
        self.L, self.H, self.d, self.causal = L, H, d, causal

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.cqsa_plan_destroy(self.handle)
            self.handle = None

    @property
    def depth(self):
        return lib().cqsa_plan_depth(self.handle)

    @property
    def num_tasks(self):
        return lib().cqsa_plan_num_tasks(self.handle)

    @property
    def modelled_device_bytes(self):
        return lib().cqsa_plan_modelled_device_bytes(self.handle)

    @property
    def tasks_per_slot(self):
        return lib().cqsa_plan_tasks_per_slot(self.handle)

    @property
    def bwd_tasks_per_launch(self):
        return lib().cqsa_plan_bwd_tasks_per_launch(self.handle)

    @property
    def acc_on_device(self):
        return lib().cqsa_plan_acc_on_device(self.handle)

    @property
    def reads_in_place(self):
        return lib().cqsa_plan_reads_in_place(self.handle)

    def task(self, t):
        """Task t as a dict of plain Python values."""
        tk = cqsa_task()
        _check(lib().cqsa_plan_get_task(self.handle, t, ctypes.byref(tk)), "cqsa_plan_get_task")
        return dict(index=tk.index, depth=tk.depth,
                    quorum=tuple(tk.quorum[i] for i in range(tk.depth)),
                    L_local=tk.L_local,
                    runs=[(tk.runs[i].global_start, tk.runs[i].length, tk.runs[i].bits)
                          for i in range(tk.n_runs)],
                    block_or=[tk.block_or[i] for i in range(tk.n_blocks)],
                    block_and=[tk.block_and[i] for i in range(tk.n_blocks)])

    def tile_census(self):
        f, c, m = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        _check(lib().cqsa_plan_tile_census(self.handle, ctypes.byref(f), ctypes.byref(c),
                                           ctypes.byref(m)), "cqsa_plan_tile_census")
        return f.value, c.value, m.value

    def fwd_tile_decisions(self):
        """(masked, clear, mixed) the inner forward's tile decisions should
        count (cqsa_plan_fwd_tile_decisions)."""
        f, c, m = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        _check(lib().cqsa_plan_fwd_tile_decisions(self.handle, ctypes.byref(f), ctypes.byref(c),
                                                  ctypes.byref(m)), "cqsa_plan_fwd_tile_decisions")
        return f.value, c.value, m.value

    def bwd_tile_decisions(self):
        """((dQ masked, clear, mixed), (dK/dV masked, clear, mixed)) the
        backward kernels' tile decisions should count
        (cqsa_plan_bwd_tile_decisions)."""
        dq, kv = (ctypes.c_int64 * 3)(), (ctypes.c_int64 * 3)()
        _check(lib().cqsa_plan_bwd_tile_decisions(self.handle, dq, kv), "cqsa_plan_bwd_tile_decisions")
        return tuple(dq), tuple(kv)


def cqsa_bwd_kv_query_tile(d):
    """Query rows of one dK/dV tile at head dim d (cqsa_bwd_kv_query_tile)."""
    return lib().cqsa_bwd_kv_query_tile(d)


def cqsa_plan(L, H, d, causal, device_budget_bytes=0, opts=None):
    """Plan a call (host only).  opts: a cqsa_plan_opts (make_opts) or None."""
    h = ctypes.c_void_p()
    po = ctypes.byref(opts) if opts is not None else None
    _check(lib().cqsa_plan(L, H, d, int(bool(causal)), int(device_budget_bytes), po,
                           ctypes.byref(h)), "cqsa_plan")
    return Plan(h.value, opts if opts is not None else cqsa_plan_opts_default(), L, H, d, causal)


# ---------------------------------------------------------------- torch glue
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _dtype_code(t):
    torch = _torch()
    return {torch.float32: CQSA_F32, torch.float16: CQSA_F16, torch.bfloat16: CQSA_BF16}[t.dtype]


def as_cqsa_tensor(t):
    """Describe a contiguous [B, L, H, d] torch tensor (no copy)."""
    if t.dim() != 4:
        raise ValueError("tensors must be [B, L, H, d]")
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return cqsa_tensor(t.data_ptr(), _dtype_code(t),
                       CQSA_MEM_DEVICE if t.is_cuda else CQSA_MEM_HOST, *t.shape)


def _stream_of(*ts):
    torch = _torch()
    for t in ts:
        if t is not None and t.is_cuda:
            return ctypes.c_void_p(torch.cuda.current_stream(t.device).cuda_stream)
    return ctypes.c_void_p(0)


def _check_lse(plan, LSE, O):
    """The C ABI takes LSE as a bare float pointer: its shape, dtype, layout and
    residency are checked here, before any call."""
    if LSE.dtype != _torch().float32 or not LSE.is_contiguous():
        raise ValueError("LSE must be a contiguous float32 tensor")
    want = (plan.opts.B, plan.H, plan.L)
    if tuple(LSE.shape) != want:
        raise ValueError(f"LSE must have shape (B, H, L) = {want}, got {tuple(LSE.shape)}")
    if LSE.is_cuda != O.is_cuda or (LSE.is_cuda and LSE.device != O.device):
        raise ValueError("LSE must live where O lives")


def cqsa_forward(plan, Q, K, V, O, LSE, scale=0.0, stream=None):
    """O (fp32 [B,L,H,d], or the input dtype with out16) and LSE (fp32 [B,H,L]) are
    written in place."""
    _check_lse(plan, LSE, O)
    tq, tk, tv, to = (as_cqsa_tensor(x) for x in (Q, K, V, O))
    s = stream if stream is not None else _stream_of(O, Q)
    _check(lib().cqsa_forward(plan.handle, ctypes.byref(tq), ctypes.byref(tk), ctypes.byref(tv),
                              ctypes.byref(to), ctypes.c_void_p(LSE.data_ptr()),
                              CQSA_MEM_DEVICE if LSE.is_cuda else CQSA_MEM_HOST,
                              float(scale), s), "cqsa_forward")


def cqsa_forward_noalloc(plan, Q, K, V, O, LSE, scale=0.0, stream=None):
    """cqsa_forward working in the device's fixed scratch array: allocates
    nothing (for graph capture and serving loops); see include/cqsa.h for its
    limits."""
    _check_lse(plan, LSE, O)
    tq, tk, tv, to = (as_cqsa_tensor(x) for x in (Q, K, V, O))
    s = stream if stream is not None else _stream_of(O, Q)
    _check(lib().cqsa_forward_noalloc(plan.handle, ctypes.byref(tq), ctypes.byref(tk),
                                      ctypes.byref(tv), ctypes.byref(to),
                                      ctypes.c_void_p(LSE.data_ptr()),
                                      CQSA_MEM_DEVICE if LSE.is_cuda else CQSA_MEM_HOST,
                                      float(scale), s), "cqsa_forward_noalloc")


def cqsa_backward(plan, Q, K, V, O, LSE, dO, dQ, dK, dV, scale=0.0, stream=None):
    """dQ, dK, dV (fp32 [B,L,H,d]) are overwritten.  Q, K, V, dO live where the
    plan's inputs do; O, LSE, dQ, dK, dV where its accumulator does."""
    _check_lse(plan, LSE, O)
    ts = [as_cqsa_tensor(x) for x in (Q, K, V, O, dO, dQ, dK, dV)]
    s = stream if stream is not None else _stream_of(dQ, Q)
    _check(lib().cqsa_backward(plan.handle, *(ctypes.byref(t) for t in ts[:4]),
                               ctypes.c_void_p(LSE.data_ptr()),
                               CQSA_MEM_DEVICE if LSE.is_cuda else CQSA_MEM_HOST,
                               *(ctypes.byref(t) for t in ts[4:]), float(scale), s),
           "cqsa_backward")


# ------------------------------------------- rotary positions, 4-bit cache
# The calls of the operators: a step of decoding makes several of a few
# microseconds each, so views are packed straight into cqsa_view's bytes (a
# third of a ctypes structure's time).
_VIEW = struct.Struct("=Qi4x7q")
_WEIGHTS = struct.Struct("=Q5q")
_PROBS = struct.Struct("=Qi4x5q")
_calls = {}


def _call(name):
    """The library's function, with the cqsa_view, cqsa_weights and cqsa_probs arguments as bytes."""
    f = _calls.get(name)
    if f is None:
        res, args = _SIGS[name]
        lib()
        f = ctypes.CDLL(LIB_PATH)[name]
        f.restype, f.argtypes = res, [ctypes.c_char_p if x in (_V, _W, _P) else x for x in args]
        _calls[name] = f
    return f


def _view(t, device):
    """The bytes of t's cqsa_view; t must live on `device`."""
    if t.device != device:
        raise ValueError("all tensors of a call must live on one device")
    s, n = t.stride(), t.shape
    if len(s) != 4:
        raise ValueError("tensors must be [B, L, H, d]")
    if s[3] != 1:
        raise ValueError("the last dimension must be contiguous")
    code = (_dtype_table or _dtypes()).get(t.dtype)
    if code is None:
        raise ValueError(f"tensors must be float32, float16 or bfloat16, got {t.dtype}")
    return _VIEW.pack(t.data_ptr(), code, n[0], n[1], n[2], n[3], s[0], s[1], s[2])


_dtype_table = {}


def _dtypes():
    if not _dtype_table:
        torch = _torch()
        _dtype_table.update({torch.float32: CQSA_F32, torch.float16: CQSA_F16, torch.bfloat16: CQSA_BF16})
    return _dtype_table


def _device_array(t, name, shape):
    """An int32 array that the C ABI takes as a bare pointer."""
    if t.dtype != _torch().int32 or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor on a GPU")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {shape}, got {tuple(t.shape)}")


def _int32(**sizes):
    """Refuse sizes that a field of 32 bits would cut off."""
    for name, x in sizes.items():
        if not 0 <= x < 2 ** 31:
            raise ValueError(f"{name} must be in [0, 2^31), got {x}")


_short = None


def _short_calls():
    """The current device's index and the current stream (an integer) of a device by its index: torch's
    own short ways where it has them (they save 2 us of every call), else by its objects."""
    global _short
    if _short is None:
        torch = _torch()
        _short = (getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device,
                  getattr(torch._C, "_cuda_getCurrentRawStream", None) or
                  (lambda i: torch.cuda.current_stream(i).cuda_stream))
    return _short


def _enqueue(name, device, stream, *args):
    """The call `name` with `device` current, on `stream` or the device's current one."""
    current_device, current_stream = _short or _short_calls()
    index = device.index
    if index != current_device():
        with _torch().cuda.device(device):
            return _enqueue(name, device, stream, *args)
    if stream is None:
        stream = current_stream(index)
    status = (_calls.get(name) or _call(name))(*args, stream)
    if status != 0:
        _check(status, name)


class RotaryPlan:
    """Owner of a cqsa_rotary_t*."""

    def __init__(self, handle, opts):
        self.handle, self.opts = handle, opts

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.cqsa_rotary_destroy(self.handle)
            self.handle = None


def cqsa_rotary_plan(d, sections=None, theta=10000.0, pairs="half", spectrum="shared", dealt=False,
                     pos_scale=None):
    """The table of a rotation (host only).  sections: pairs of each axis (None:
    one axis, all d / 2); pairs: "half" or "adjacent"; spectrum: "shared" or
    "per_axis"; dealt: pairs dealt to the axes in turn; pos_scale: a factor of
    each axis's positions."""
    o = cqsa_rotary_opts()
    if d >= 2 ** 31 or any(n >= 2 ** 31 for n in sections or ()):
        raise ValueError("d and the sections must be below 2^31")
    lib().cqsa_rotary_opts_default(ctypes.byref(o), d)
    o.pairs = {"half": 0, "adjacent": 1}[pairs]
    o.spectrum = {"shared": 0, "per_axis": 1}[spectrum]
    o.dealt, o.theta = int(bool(dealt)), theta
    if sections is not None:
        if len(sections) > 4:
            raise ValueError("at most 4 axes")
        o.n_axes = len(sections)
        for a, n in enumerate(sections):
            o.sections[a] = n
    if pos_scale is not None:
        if len(pos_scale) != o.n_axes:
            raise ValueError("pos_scale needs a factor for each axis")
        for a, f in enumerate(pos_scale):
            o.pos_scale[a] = f
    h = ctypes.c_void_p()
    _check(lib().cqsa_rotary_plan(ctypes.byref(o), ctypes.byref(h)), "cqsa_rotary_plan")
    return RotaryPlan(h.value, o)


def cqsa_rotary(plan, pos, x, y=None, inverse=False, stream=None):
    """Turn x (a [B, L, H, d] tensor, or a list of one or two: Q, or Q and K)
    into y (None: in place) by positions pos, int32 [axes, B, L].  inverse=True
    gives the gradient of x from that of y."""
    xs = (x,) if hasattr(x, "data_ptr") else x
    ys = xs if y is None else (y,) if hasattr(y, "data_ptr") else y
    n = len(xs)
    if n not in (1, 2) or len(ys) != n:
        raise ValueError("one or two tensors, and as many results")
    shape = xs[0].shape
    _device_array(pos, "pos", (plan.opts.n_axes, shape[0], shape[1]))
    device = pos.device
    vx = b"".join([_view(t, device) for t in xs])
    vy = vx if ys is xs else b"".join([_view(t, device) for t in ys])
    _enqueue("cqsa_rotary", device, stream, plan.handle, pos.data_ptr(), vx, vy, n, 1 if inverse else 0)


def cqsa_cache_page_bytes(page_size, H, d):
    """Bytes of one page of the 4-bit cache (cqsa_cache_page_bytes)."""
    return lib().cqsa_cache_page_bytes(page_size, H, d)


class _Fixed:
    """Made once: the C structure of a call holds the addresses of its tensors, whose
    contents may change, but which no others can replace."""

    def __setattr__(self, name, value):
        raise AttributeError(f"a {type(self).__name__} is made once; make another, or copy into its tensors")


class Cache4(_Fixed):
    """A paged 4-bit cache of keys and values (cqsa_cache): n_pages pages of
    page_size tokens of H heads.  data: a contiguous uint8 tensor to keep it in
    (None: a new one of zeros on `device`)."""

    def __init__(self, n_pages, H, d, page_size=64, data=None, device="cuda"):
        torch = _torch()
        _int32(page_size=page_size, H=H, d=d)
        per = cqsa_cache_page_bytes(page_size, H, d)
        if per == 0:
            raise ValueError("page_size must be 32, 64, 128 or 256, H in [1, 65536], "
                             "d a multiple of 32 in [32, 256]")
        if data is None:
            data = torch.zeros((n_pages, per), dtype=torch.uint8, device=device)
        if data.dtype != torch.uint8 or not data.is_cuda or not data.is_contiguous():
            raise ValueError("data must be a contiguous uint8 tensor on a GPU")
        if data.numel() != n_pages * per:
            raise ValueError(f"data must have {n_pages} x {per} bytes")
        self.__dict__.update(n_pages=n_pages, H=H, d=d, page_size=page_size, data=data, device=data.device,
                             view=cqsa_cache(data.data_ptr(), n_pages, page_size, H, d))


class CacheBatch(_Fixed):
    """The sequences of a call (cqsa_cache_batch).  pages: int32 [B, max_pages];
    lengths: int32 [B], the tokens in the cache with the call's; q_start: int32
    [B + 1] for packed rows, then max_q bounds a sequence's rows (0: all that the
    tensors have; the launch goes by it, so single tokens want max_q=1).  max_len
    bounds the lengths (0: the table's tokens, once a cache says how many)."""

    def __init__(self, pages, lengths, q_start=None, max_len=0, max_q=0):
        _int32(max_len=max_len, max_q=max_q)
        if pages.dim() != 2 or pages.dtype != _torch().int32 or not pages.is_cuda or \
                (pages.shape[1] > 1 and pages.stride(1) != 1):
            raise ValueError("pages must be an int32 tensor [B, max_pages] on a GPU with contiguous rows")
        B, n = pages.shape
        _device_array(lengths, "lengths", (B,))
        if q_start is not None:
            _device_array(q_start, "q_start", (B + 1,))
        device = pages.device
        if lengths.device != device or (q_start is not None and q_start.device != device):
            raise ValueError("all tensors of a batch must live on one device")
        view = cqsa_cache_batch(pages.data_ptr(), pages.stride(0) if B > 1 else n, lengths.data_ptr(),
                                q_start.data_ptr() if q_start is not None else None, B, n, max_len, max_q)
        self.__dict__.update(pages=pages, lengths=lengths, q_start=q_start, max_len=max_len, max_q=max_q,
                             device=device, view=view)

    def _bound(self, cache):
        """The descriptor for a cache, without rows: a bound on the lengths left open filled in."""
        if self.max_len:
            return self.view
        v = cqsa_cache_batch.from_buffer_copy(self.view)
        v.max_len = min(v.max_pages * cache.page_size, 2 ** 30)
        return v

    def _of(self, cache, t):
        """The descriptor for a cache and a tensor of rows: the bounds left open filled in."""
        v = self._bound(cache)
        if self.max_q or self.q_start is None:
            return v
        if v is self.view:
            v = cqsa_cache_batch.from_buffer_copy(v)
        v.max_q = t.shape[1]
        return v


def _cache_device(cache, batch):
    if cache.device != batch.device:
        raise ValueError("the cache and the batch must live on one device")
    return cache.device


def _cache_move(name, cache, batch, K, V, stream):
    device = _cache_device(cache, batch)
    _enqueue(name, device, stream, cache.view, batch._of(cache, K), _view(K, device), _view(V, device))


def cqsa_cache_write(cache, batch, K, V, stream=None):
    """Quantise the call's rows of K and V into the cache's pages."""
    _cache_move("cqsa_cache_write", cache, batch, K, V, stream)


def cqsa_cache_read(cache, batch, K, V, stream=None):
    """Fill K and V with the values that the cache holds for the call's rows."""
    _cache_move("cqsa_cache_read", cache, batch, K, V, stream)


def cqsa_cache_attend_workspace(cache, batch, Q):
    """A workspace for cqsa_cache_attend with arguments of these sizes (a uint8
    tensor, or None where none is needed); calls that may overlap need their own."""
    n = ctypes.c_uint64()
    device = _cache_device(cache, batch)
    _check(_call("cqsa_cache_attend_workspace")(cache.view, batch._of(cache, Q), _view(Q, device), n),
           "cqsa_cache_attend_workspace")
    return _torch().empty(n.value, dtype=_torch().uint8, device=device) if n.value else None


def cqsa_cache_attend_launch(cache, batch, Q):
    """How cqsa_cache_attend launches a call with arguments of these sizes
    (cqsa_attend_launch: many, rows, waves, splits)."""
    out = cqsa_attend_launch()
    _check(_call("cqsa_cache_attend_launch")(cache.view, batch._of(cache, Q), _view(Q, _cache_device(cache, batch)), out),
           "cqsa_cache_attend_launch")
    return out


def _workspace_on(stream, device, make, *args):
    """make(*args), a workspace from torch's allocator, for one call on `stream` (None: the current one)."""
    if stream is None:
        return make(*args)
    cuda = _torch().cuda
    handle = getattr(stream, "value", stream) or 0
    with cuda.stream(cuda.ExternalStream(handle, device=device) if handle else cuda.default_stream(device)):
        return make(*args)


def _place(workspace, device):
    """The address and size of a workspace, or (None, 0)."""
    if workspace is None:
        return None, 0
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"the workspace must be a contiguous tensor on {device}")
    return workspace.data_ptr(), workspace.nbytes


def _lse(LSE, Q, device):
    """The address of an LSE for the rows of Q."""
    B, L, H, _ = Q.shape
    if LSE is None or LSE.dtype is not _torch().float32 or LSE.device != device or not LSE.is_contiguous() or LSE.shape != (B, H, L):
        raise ValueError(f"LSE must be a contiguous float32 tensor of shape (B, H, L) = {(B, H, L)} on {device}")
    return LSE.data_ptr()


def cqsa_cache_attend(cache, batch, Q, O, LSE=None, causal=True, scale=0.0, workspace=None, stream=None):
    """Attention of the call's rows Q over their sequences' cached tokens into O
    and, if given, LSE (fp32 [B, Hq, L], packed [1, Hq, T]).  workspace=None
    takes one from torch's allocator for this call and its stream."""
    device = _cache_device(cache, batch)
    vq, vo = _view(Q, device), _view(O, device)
    lse = None if LSE is None else _lse(LSE, Q, device)
    if workspace is None:
        workspace = _workspace_on(stream, device, cqsa_cache_attend_workspace, cache, batch, Q)
    space, size = _place(workspace, device)
    _enqueue("cqsa_cache_attend", device, stream, cache.view, batch._of(cache, Q), vq, vo, lse,
             1 if causal else 0, scale, space, size)


# ------------------------------- cached tokens' weights, eviction, drafted tokens
def _weights(t, name, device):
    """The bytes of t's cqsa_weights."""
    s, n = (t.stride(), t.shape) if t is not None else ((), ())
    if len(s) != 3 or t.dtype is not _torch().float32 or t.device != device or (s[2] != 1 and n[2] > 1):
        raise ValueError(f"{name} must be a float32 tensor [B, H, T] on {device} with contiguous tokens")
    return _WEIGHTS.pack(t.data_ptr(), *n, s[0], s[1])


def _ints(t, name, shape, device):
    """The address of an int32 array, or None."""
    if t is None:
        return None
    if t.dtype is not _torch().int32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous int32 tensor of shape {shape} on {device}")
    return t.data_ptr()


def cqsa_cache_weigh_workspace(cache, batch, Q):
    """A workspace for cqsa_cache_weigh with arguments of these sizes (a uint8 tensor, or
    None where none is needed); calls that may overlap need their own."""
    n = ctypes.c_uint64()
    device = _cache_device(cache, batch)
    _check(_call("cqsa_cache_weigh_workspace")(cache.view, batch._of(cache, Q), _view(Q, device), n),
           "cqsa_cache_weigh_workspace")
    return _torch().empty(n.value, dtype=_torch().uint8, device=device) if n.value else None


def cqsa_cache_weigh(cache, batch, Q, LSE, W, prior=None, decay=1.0, counts=None, causal=True, scale=0.0,
                     workspace=None, stream=None):
    """W (fp32 [B, H, T >= max_len]) at each cached token: decay times prior (None: 0, may be
    W; the rows' own tokens start from 0) and the sum of the attention weights that the call's
    rows Q give it, LSE (fp32 [B, Hq, L]) being what cqsa_cache_attend left for them.  counts
    (int32 [B]): only the first counts[b] rows of sequence b."""
    device = _cache_device(cache, batch)
    q, w = _view(Q, device), _weights(W, "W", device)
    old = w if prior is W else None if prior is None else _weights(prior, "prior", device)
    lse = _lse(LSE, Q, device)
    n = None if counts is None else _ints(counts, "counts", (batch.view.B,), device)
    if workspace is None:
        workspace = _workspace_on(stream, device, cqsa_cache_weigh_workspace, cache, batch, Q)
    space, size = _place(workspace, device)
    _enqueue("cqsa_cache_weigh", device, stream, cache.view, batch._of(cache, Q), q, lse, n, old, decay, w,
             1 if causal else 0, scale, space, size)


def _tables(to, batch, device):
    """The cqsa_cache_batch of a target's page tables."""
    if to.dim() != 2 or to.dtype != _torch().int32 or to.device != device or (to.shape[1] > 1 and to.stride(1) != 1):
        raise ValueError(f"to must be an int32 tensor [B, max_pages] on {device} with contiguous rows")
    B, n = to.shape
    if B != batch.view.B:
        raise ValueError("to must have a table for each of the batch's sequences")
    return cqsa_cache_batch(to.data_ptr(), to.stride(0) if B > 1 else n, None, None, B, n, 0, 0)


def cqsa_cache_evict_workspace(cache, batch, budget, to=None):
    """A workspace for cqsa_cache_evict with arguments of these sizes (a uint8 tensor)."""
    n = ctypes.c_uint64()
    _int32(budget=budget)
    device = _cache_device(cache, batch)
    _check(_call("cqsa_cache_evict_workspace")(cache.view, batch._bound(cache), budget, 1 if to is None else 0, n),
           "cqsa_cache_evict_workspace")
    return _torch().empty(n.value, dtype=_torch().uint8, device=device) if n.value else None


def cqsa_cache_evict(cache, batch, W, new_lengths, budget, first=0, recent=0, to=None, W_to=None, kept=None,
                     workspace=None, stream=None):
    """Keep, for each head of each sequence, its `first` and `recent` tokens and of the others
    those of most weight W (fp32 [B, H, T]), `budget` in all, moved together: in place, or into
    the pages of the tables `to` (int32 [B, max_pages]) with their weights in W_to.
    new_lengths (int32 [B], may be the batch's lengths) and kept (int32 [B, H, budget] or None: the
    positions they had, -1 behind them) are written."""
    device = _cache_device(cache, batch)
    _int32(budget=budget, first=first, recent=recent)
    w = _weights(W, "W", device)
    w_to = None if W_to is None else _weights(W_to, "W_to", device)
    B = batch.view.B
    at = _ints(kept, "kept", (B, cache.H, budget), device)
    new = _ints(new_lengths, "new_lengths", (B,), device)
    tables = None if to is None else _tables(to, batch, device)
    if workspace is None:
        workspace = _workspace_on(stream, device, cqsa_cache_evict_workspace, cache, batch, budget, to)
    space, size = _place(workspace, device)
    _enqueue("cqsa_cache_evict", device, stream, cache.view, batch._bound(cache), w,
             cqsa_evict_opts(budget, first, recent), tables, w_to, at, new, space, size)


def _probs(t, name, device):
    """The bytes of t's cqsa_probs."""
    s, n = (t.stride(), t.shape) if t is not None else ((), ())
    code = (_dtype_table or _dtypes()).get(t.dtype) if len(s) == 3 else None
    if code is None or t.device != device or (n[2] > 1 and s[2] != 1):
        raise ValueError(f"{name} must be a float32, float16 or bfloat16 tensor [B, rows, V] on {device} with "
                         "contiguous rows")
    return _PROBS.pack(t.data_ptr(), code, *n, s[0], s[1])


def cqsa_draft_verify_workspace(target, draft=None):
    """A workspace for cqsa_draft_verify with arguments of these sizes (a uint8 tensor, or
    None where none is needed); calls that may overlap need their own."""
    n = ctypes.c_uint64()
    _check(_call("cqsa_draft_verify_workspace")(_probs(target, "target", target.device), n),
           "cqsa_draft_verify_workspace")
    return _torch().empty(n.value, dtype=_torch().uint8, device=target.device) if n.value else None


def cqsa_draft_verify(target, draft, tokens, u, out, n_out, counts=None, lengths=None, new_lengths=None,
                      workspace=None, stream=None):
    """Accept drafted tokens (int32 [B, K]) against the target's probabilities [B, K + 1, V] and
    the draft's [B, K, V] (None: tokens that come without), by random numbers u (fp32 [B, K + 1] in
    [0, 1)), and draw the token behind the accepted ones.  out (int32 [B, K + 1]) gets them, -1 behind, n_out
    (int32 [B]) how many; new_lengths those of the cache without the refused ones' rows."""
    if target is None or not target.is_cuda:
        raise ValueError("target must live on a GPU")
    device = target.device
    p = _probs(target, "target", device)
    q = None if draft is None else _probs(draft, "draft", device)
    B, K = target.shape[0], target.shape[1] - 1
    if u is None or u.dtype != _torch().float32 or u.device != device or not u.is_contiguous() or u.shape != (B, K + 1):
        raise ValueError(f"u must be a contiguous float32 tensor of shape {(B, K + 1)} on {device}")
    one, few = (B,), (B, K + 1)
    tokens, counts = _ints(tokens, "tokens", (B, K), device), _ints(counts, "counts", one, device)
    out, n_out = _ints(out, "out", few, device), _ints(n_out, "n_out", one, device)
    lengths, new_lengths = _ints(lengths, "lengths", one, device), _ints(new_lengths, "new_lengths", one, device)
    if workspace is None:
        workspace = _workspace_on(stream, device, cqsa_draft_verify_workspace, target)
    space, size = _place(workspace, device)
    _enqueue("cqsa_draft_verify", device, stream, p, q, tokens, counts, u.data_ptr(), out, n_out, lengths, new_lengths,
             space, size)


def cqsa_set_timing(enable):
    _check(lib().cqsa_set_timing(int(bool(enable))), "cqsa_set_timing")


def cqsa_set_tile_counting(enable):
    _check(lib().cqsa_set_tile_counting(int(bool(enable))), "cqsa_set_tile_counting")


def cqsa_last_stats():
    st = cqsa_run_stats()
    _check(lib().cqsa_last_stats(ctypes.byref(st)), "cqsa_last_stats")
    return {name: getattr(st, name) for name, _ in cqsa_run_stats._fields_}


def cqsa_release_workspace():
    _check(lib().cqsa_release_workspace(), "cqsa_release_workspace")


_ALLOC_FN = ctypes.CFUNCTYPE(ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p)
_RELEASE_FN = ctypes.CFUNCTYPE(None, ctypes.c_void_p, ctypes.c_void_p)
_hooks = None  # the installed callbacks, kept alive while the library may call them


def cqsa_set_allocator(alloc=None, release=None):
    """Route the library's device workspace through alloc(nbytes) -> int device
    address (0 = failure) and release(address); None for both restores the
    built-in cached workspace."""
    global _hooks
    if (alloc is None) != (release is None):
        raise ValueError("give both functions or neither")
    if alloc is None:
        _check(lib().cqsa_set_allocator(None, None, None), "cqsa_set_allocator")
        _hooks = None
        return
    a = _ALLOC_FN(lambda n, ctx: alloc(int(n)) or None)
    r = _RELEASE_FN(lambda ptr, ctx: release(int(ptr)))
    _check(lib().cqsa_set_allocator(ctypes.cast(a, ctypes.c_void_p), ctypes.cast(r, ctypes.c_void_p),
                                    None), "cqsa_set_allocator")
    _hooks = (a, r)


def use_torch_allocator(device=None):
    """Serve the workspace from torch's caching allocator (on `device`)."""
    torch = _torch()
    held = {}

    def alloc(n):
        t = torch.empty((n,), dtype=torch.uint8, device=device or "cuda")
        held[t.data_ptr()] = t
        return t.data_ptr()

    def release(ptr):
        held.pop(ptr, None)

    cqsa_set_allocator(alloc, release)
    return held


def forward(Q, K, V, causal, device_budget_bytes=0, depth=-1, scale=0.0, **opt_kw):
    """Plan and run a forward; returns (O, LSE, plan).  Outputs live where Q lives
    unless acc_on_device is given."""
    torch = _torch()
    B, L, H, d = Q.shape
    dt = {torch.float32: "f32", torch.float16: "f16", torch.bfloat16: "bf16"}[Q.dtype]
    opt_kw.setdefault("inputs_on_device", Q.is_cuda)
    opt_kw.setdefault("acc_on_device", Q.is_cuda)
    opts = make_opts(B=B, dtype=dt, depth=depth, **opt_kw)
    plan = cqsa_plan(L, H, d, causal, device_budget_bytes, opts)
    dev = Q.device if opts.acc_on_device else torch.device("cpu")
    pin = not opts.acc_on_device and torch.cuda.is_available()
    O = torch.empty((B, L, H, d), dtype=torch.float32, device=dev, pin_memory=pin)
    LSE = torch.empty((B, H, L), dtype=torch.float32, device=dev, pin_memory=pin)
    cqsa_forward(plan, Q, K, V, O, LSE, scale)
    return O, LSE, plan
