"""ctypes binding of libflexattn.so (include/flexattn.h).

Argument marshalling only: every step of the attention path runs in the HIP
library. PyTorch supplies device memory and streams. Importing this module
raises if the library has not been built; there is no fallback.

Functions keep the C names (``flex_attn_plan``, ``flex_attn_decode``, ...);
``PagedAttention`` bundles a plan with its device copy and workspace for the
common case of running one batch.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libflexattn.so")

FLEX_OK = 0
FLEX_ERR_INVALID_ARG = -1
FLEX_ERR_UNSUPPORTED = -2
FLEX_ERR_WORKSPACE = -3
FLEX_ERR_HIP = -4
FLEX_ERR_INTERNAL = -5
FLEX_MODE_SERIAL = 0
FLEX_MODE_CORUN = 1
FLEX_MODE_FUSED = 2

EXPORTED = [
    "flex_attn_status_string", "flex_attn_last_error", "flex_attn_plan", "flex_attn_plan_info_get",
    "flex_attn_plan_export", "flex_attn_plan_upload", "flex_attn_plan_destroy", "flex_attn_decode",
    "flex_attn_prefill", "flex_attn_mixed", "flex_attn_corun_create", "flex_attn_corun_destroy",
    "flex_attn_corun_streams", "flex_attn_corun_set_timing", "flex_attn_corun_timing_read",
    "flex_attn_debug_gather", "flex_attn_workspace_init", "flex_attn_kv_append",
    "flex_attn_mixed_static", "flex_attn_static_scratch_bytes", "flex_attn_validate_host", "flex_attn_set_debug",
    "flex_attn_rope_append", "flex_attn_kv8_append", "flex_attn_decode_kv8", "flex_attn_prefill_kv8",
    "flex_attn_mixed_kv8",
    "flex_ctl_create", "flex_ctl_destroy", "flex_ctl_set_profile", "flex_ctl_observe", "flex_ctl_decide",
    "flex_ctl_estimates", "flex_ts_create", "flex_ts_destroy", "flex_ts_next", "flex_ts_observe", "flex_ts_totals",
]
FLEX_CTL_ONE_PHASE = 0
FLEX_CTL_BEST = 1
FLEX_CTL_SERIAL_FASTER = 2
FLEX_CTL_BACKLOG = 3
FLEX_CTL_BW_SATURATED = 4
FLEX_CTL_EXPLORE = 5
FLEX_CTL_PREFILL_BACKLOG = 6
FLEX_CTL_FUSED_FASTER = 7
FLEX_TS_DECODE = 0
FLEX_TS_PREFILL = 1
FLEX_TIMING_RING = 1024
FLEX_ROPE_MAX_AXES = 4


class Shape(ctypes.Structure):
    _fields_ = [("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32),
                ("head_dim_qk", ctypes.c_int32), ("head_dim_v", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("sm_scale", ctypes.c_float),
                ("v_aliases_k", ctypes.c_int32)]


class PlanOpts(ctypes.Structure):
    _fields_ = [("cus_total", ctypes.c_int32), ("cus_decode", ctypes.c_int32), ("bm", ctypes.c_int32),
                ("min_split_tokens", ctypes.c_int32),
                ("wg_per_cu", ctypes.c_int32), ("split_granule", ctypes.c_int32),
                ("hbm_gbps", ctypes.c_double), ("decode_gbps_per_cu", ctypes.c_double),
                ("prefill_tflops_per_cu", ctypes.c_double), ("decode_tail", ctypes.c_int32),
                ("kv_bits", ctypes.c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32), ("n_decode_seqs", ctypes.c_int32),
                ("n_prefill_seqs", ctypes.c_int32), ("n_decode_items", ctypes.c_int32),
                ("n_prefill_items", ctypes.c_int32), ("n_split_seqs", ctypes.c_int32),
                ("decode_wg_width", ctypes.c_int32), ("n_decode_ranges", ctypes.c_int32),
                ("prefill_grid_y", ctypes.c_int32), ("pages_per_split", ctypes.c_int32),
                ("cus_decode", ctypes.c_int32), ("cus_prefill", ctypes.c_int32), ("bm", ctypes.c_int32),
                ("plan_words", ctypes.c_int32), ("device_plan_bytes", ctypes.c_size_t),
                ("workspace_bytes", ctypes.c_size_t), ("decode_bytes", ctypes.c_double),
                ("prefill_flops", ctypes.c_double), ("n_fused_wgs", ctypes.c_int32),
                ("n_decode_tail_ranges", ctypes.c_int32), ("decode_tail_bytes", ctypes.c_double)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class Args(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k_cache", ctypes.c_void_p), ("v_cache", ctypes.c_void_p),
                ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
                ("num_pages", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("block_table_stride", ctypes.c_int32), ("seq_lens", ctypes.c_void_p),
                ("query_start_loc", ctypes.c_void_p), ("out", ctypes.c_void_p), ("lse", ctypes.c_void_p),
                ("d_plan", ctypes.c_void_p), ("d_plan_bytes", ctypes.c_size_t),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


class AppendArgs(ctypes.Structure):
    _fields_ = [("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("k_new_stride", ctypes.c_int64),
                ("v_new_stride", ctypes.c_int64), ("slot_mapping", ctypes.c_void_p), ("n_tokens", ctypes.c_int64),
                ("k_cache", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3), ("v_cache", ctypes.c_void_p),
                ("v_stride", ctypes.c_int64 * 3), ("num_pages", ctypes.c_int64), ("bad_count", ctypes.c_void_p)]


class Rope(ctypes.Structure):
    _fields_ = [("cos_sin", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_stride", ctypes.c_int64),
                ("max_position", ctypes.c_int32), ("rot_begin", ctypes.c_int32), ("rot_dim", ctypes.c_int32),
                ("neighbours", ctypes.c_int32), ("n_axes", ctypes.c_int32), ("dealt", ctypes.c_int32),
                ("sections", ctypes.c_int32 * FLEX_ROPE_MAX_AXES)]


class RopeAppendArgs(ctypes.Structure):
    _fields_ = [("kv", AppendArgs), ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("q_out", ctypes.c_void_p)]


class Kv8AppendArgs(ctypes.Structure):
    _fields_ = [("k_new", ctypes.c_void_p), ("v_new", ctypes.c_void_p), ("k_new_stride", ctypes.c_int64),
                ("v_new_stride", ctypes.c_int64), ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64),
                ("q_out", ctypes.c_void_p), ("n_tokens", ctypes.c_int64), ("num_seqs", ctypes.c_int32),
                ("block_table", ctypes.c_void_p), ("block_table_stride", ctypes.c_int32),
                ("seq_lens", ctypes.c_void_p), ("query_start_loc", ctypes.c_void_p), ("k_cache", ctypes.c_void_p),
                ("k_stride", ctypes.c_int64 * 3), ("v_cache", ctypes.c_void_p), ("v_stride", ctypes.c_int64 * 3),
                ("kv_scales", ctypes.c_void_p), ("scale_page_stride", ctypes.c_int64),
                ("num_pages", ctypes.c_int64), ("bad_count", ctypes.c_void_p)]


class Kv8Args(ctypes.Structure):
    _fields_ = [("attn", Args), ("kv_scales", ctypes.c_void_p), ("scale_page_stride", ctypes.c_int64)]


class CtlOpts(ctypes.Structure):
    _fields_ = [("cus_total", ctypes.c_int32), ("granule", ctypes.c_int32), ("explore_every", ctypes.c_int32),
                ("backlog_seqs", ctypes.c_int32), ("backlog_prefill_tokens", ctypes.c_int32),
                ("alpha", ctypes.c_double), ("tolerance", ctypes.c_double), ("sat_frac", ctypes.c_double),
                ("hbm_gbps", ctypes.c_double), ("corun_overhead_us", ctypes.c_double),
                ("decode_gbps_per_cu", ctypes.c_double), ("prefill_tflops_per_cu", ctypes.c_double),
                ("fused_prior", ctypes.c_double)]


class CtlSignals(ctypes.Structure):
    _fields_ = [("decode_bytes", ctypes.c_double), ("prefill_flops", ctypes.c_double),
                ("pending_prefill_tokens", ctypes.c_int32), ("pending_decode_seqs", ctypes.c_int32),
                ("active_decode_seqs", ctypes.c_int32), ("fused_available", ctypes.c_int32),
                ("decode_tail", ctypes.c_int32)]


class CtlObservation(ctypes.Structure):
    _fields_ = [("cus_decode", ctypes.c_int32), ("decode_bytes", ctypes.c_double),
                ("prefill_flops", ctypes.c_double), ("decode_ms", ctypes.c_double), ("prefill_ms", ctypes.c_double),
                ("fused", ctypes.c_int32), ("step_ms", ctypes.c_double)]


class CtlDecision(ctypes.Structure):
    _fields_ = [("mode", ctypes.c_int32), ("cus_decode", ctypes.c_int32), ("cus_prefill", ctypes.c_int32),
                ("reason", ctypes.c_int32), ("predicted_us", ctypes.c_double)]


class TsOpts(ctypes.Structure):
    _fields_ = [("decode_share", ctypes.c_double), ("decay", ctypes.c_double)]


class FlexAttnError(RuntimeError):
    def __init__(self, status: int, what: str, detail: str):
        super().__init__(f"{what}: status {status} ({detail})")
        self.status = status


_lib = None


def lib():
    """Load libflexattn.so (once). Raises if it is missing: there is no fallback."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing; build it with "
                           "`python -m paper_2606_04415_amd.build` (hipcc, gfx950)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    L.flex_attn_status_string.argtypes = [ctypes.c_int]
    L.flex_attn_status_string.restype = ctypes.c_char_p
    L.flex_attn_last_error.argtypes = []
    L.flex_attn_last_error.restype = ctypes.c_char_p
    L.flex_attn_plan.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(PlanOpts), i32,
                                 ctypes.POINTER(i32), ctypes.POINTER(i32), i32, ctypes.POINTER(vp)]
    L.flex_attn_plan_info_get.argtypes = [vp, ctypes.POINTER(PlanInfo)]
    L.flex_attn_plan_export.argtypes = [vp, ctypes.POINTER(i32), sz]
    L.flex_attn_plan_upload.argtypes = [vp, vp, sz, vp]
    L.flex_attn_plan_destroy.argtypes = [vp]
    L.flex_attn_plan_destroy.restype = None
    for f in ("flex_attn_decode", "flex_attn_prefill"):
        getattr(L, f).argtypes = [vp, ctypes.POINTER(Args), vp]
    L.flex_attn_mixed.argtypes = [vp, ctypes.POINTER(Args), ctypes.c_int, vp, vp]
    L.flex_attn_mixed_static.argtypes = [vp, ctypes.POINTER(Args), ctypes.c_int, vp, vp]
    L.flex_attn_static_scratch_bytes.argtypes = []
    L.flex_attn_static_scratch_bytes.restype = ctypes.c_size_t
    L.flex_attn_validate_host.argtypes = [vp, ctypes.POINTER(i32), i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
    L.flex_attn_set_debug.argtypes = [ctypes.c_int]
    L.flex_attn_corun_create.argtypes = [i32, i32, ctypes.POINTER(vp)]
    L.flex_attn_corun_destroy.argtypes = [vp]
    L.flex_attn_corun_destroy.restype = None
    L.flex_attn_corun_streams.argtypes = [vp, ctypes.POINTER(vp), ctypes.POINTER(vp)]
    L.flex_attn_corun_set_timing.argtypes = [vp, ctypes.c_int]
    L.flex_attn_corun_timing_read.argtypes = [vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_float),
                                              i32, ctypes.POINTER(i32)]
    L.flex_attn_debug_gather.argtypes = [vp, ctypes.POINTER(Args), i32, i32, vp, vp, vp]
    L.flex_attn_workspace_init.argtypes = [vp, sz, vp]
    L.flex_attn_kv_append.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(AppendArgs), vp]
    L.flex_attn_rope_append.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(Rope), ctypes.POINTER(RopeAppendArgs), vp]
    L.flex_attn_kv8_append.argtypes = [ctypes.POINTER(Shape), ctypes.POINTER(Rope), ctypes.POINTER(Kv8AppendArgs), vp]
    for f in ("flex_attn_decode_kv8", "flex_attn_prefill_kv8"):
        getattr(L, f).argtypes = [vp, ctypes.POINTER(Kv8Args), vp]
    L.flex_attn_mixed_kv8.argtypes = [vp, ctypes.POINTER(Kv8Args), ctypes.c_int, vp, vp]
    L.flex_ctl_create.argtypes = [ctypes.POINTER(CtlOpts), ctypes.POINTER(vp)]
    L.flex_ctl_destroy.argtypes = [vp]
    L.flex_ctl_destroy.restype = None
    L.flex_ctl_set_profile.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(ctypes.c_double)]
    L.flex_ctl_observe.argtypes = [vp, ctypes.POINTER(CtlObservation)]
    L.flex_ctl_decide.argtypes = [vp, ctypes.POINTER(CtlSignals), ctypes.POINTER(CtlDecision)]
    L.flex_ctl_estimates.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double), i32]
    L.flex_ts_create.argtypes = [ctypes.POINTER(TsOpts), ctypes.POINTER(vp)]
    L.flex_ts_destroy.argtypes = [vp]
    L.flex_ts_destroy.restype = None
    L.flex_ts_next.argtypes = [vp, i32, i32, ctypes.POINTER(i32)]
    L.flex_ts_observe.argtypes = [vp, i32, ctypes.c_double]
    L.flex_ts_totals.argtypes = [vp, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_double)]
    for f in EXPORTED:
        if f not in ("flex_attn_status_string", "flex_attn_last_error", "flex_attn_plan_destroy",
                     "flex_attn_corun_destroy", "flex_ctl_destroy", "flex_ts_destroy",
                     "flex_attn_static_scratch_bytes"):
            getattr(L, f).restype = ctypes.c_int
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().flex_attn_status_string(status).decode()


def last_error() -> str:
    return lib().flex_attn_last_error().decode()


def check(status: int, what: str):
    if status != FLEX_OK:
        raise FlexAttnError(status, what, f"{status_string(status)}: {last_error()}")


def _i32_array(values):
    """An int32* argument over values (an int sequence, a numpy array or a CPU
    tensor): a view when they already are contiguous int32, else one
    vectorised conversion (no per-element Python loop). Values outside int32
    raise ValueError. The returned pointer keeps its array alive."""
    import numpy as np
    if hasattr(values, "detach"):   # torch tensor
        values = values.detach().cpu().numpy()
    a = np.asarray(values).reshape(-1)
    if a.dtype != np.int32:
        if a.size and (a.dtype.kind not in "iu" or int(a.min()) < -2 ** 31 or int(a.max()) > 2 ** 31 - 1):
            raise ValueError("expected integers that fit int32")
        a = a.astype(np.int32)
    a = np.ascontiguousarray(a) if a.size else np.zeros(1, dtype=np.int32)
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


class Plan:
    """Owning wrapper of a flex_attn_plan_t*."""

    def __init__(self, handle: int):
        self.handle = ctypes.c_void_p(handle)
        info = PlanInfo()
        check(lib().flex_attn_plan_info_get(self.handle, ctypes.byref(info)), "flex_attn_plan_info_get")
        self.info = info.as_dict()

    def export(self):
        n = self.info["plan_words"]
        buf = (ctypes.c_int32 * n)()
        check(lib().flex_attn_plan_export(self.handle, buf, n), "flex_attn_plan_export")
        return list(buf)

    def close(self):
        if self.handle and self.handle.value:
            lib().flex_attn_plan_destroy(self.handle)
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def make_shape(num_q_heads, num_kv_heads, head_dim_qk, head_dim_v, page_size, sm_scale, v_aliases_k=False):
    return Shape(num_q_heads, num_kv_heads, head_dim_qk, head_dim_v, page_size, float(sm_scale),
                 1 if v_aliases_k else 0)


def make_opts(**kw) -> PlanOpts:
    o = PlanOpts()
    for k, v in kw.items():
        setattr(o, k, v)
    return o


def flex_attn_plan(shape: Shape, opts: Optional[PlanOpts], query_start_loc: Sequence[int],
                   seq_lens: Sequence[int], max_pages_per_seq: int) -> Plan:
    """Host plan (no HIP call). query_start_loc and seq_lens: int sequences,
    numpy arrays or CPU tensors. Raises FlexAttnError with the library's
    status on failure."""
    out = ctypes.c_void_p()
    starts = _i32_array(query_start_loc)
    st = lib().flex_attn_plan(ctypes.byref(shape), ctypes.byref(opts) if opts is not None else None,
                              len(seq_lens), starts, _i32_array(seq_lens),
                              int(max_pages_per_seq), ctypes.byref(out))
    check(st, "flex_attn_plan")
    plan = Plan(out.value)
    plan.shape = Shape.from_buffer_copy(shape)
    plan.batch = (len(seq_lens), starts[len(seq_lens)])   # (the array may go on)
    return plan


def plan_status(shape: Shape, opts: Optional[PlanOpts], query_start_loc, seq_lens, max_pages_per_seq) -> int:
    """Status code of flex_attn_plan for these inputs (the plan, if any, is freed)."""
    out = ctypes.c_void_p()
    st = lib().flex_attn_plan(ctypes.byref(shape), ctypes.byref(opts) if opts is not None else None,
                              len(seq_lens), _i32_array(query_start_loc), _i32_array(seq_lens),
                              int(max_pages_per_seq), ctypes.byref(out))
    if st == FLEX_OK:
        lib().flex_attn_plan_destroy(out)
    return st


# ------------------------------------------------------- torch adapters ---

def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def current_stream():
    import torch
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _require(cond, what):
    if not cond:
        raise ValueError(what)


def make_args(q, k_cache, v_cache, block_table, seq_lens, query_start_loc, out, lse=None,
              d_plan=None, workspace=None) -> Args:
    """Args from device tensors (bf16 caches [pages, P, Hkv, d] with unit inner stride).

    Checks what the C side cannot see: dtypes (bf16 q/caches/out, fp32 lse,
    int32 metadata), contiguity of q, out, lse and the metadata rows, a unit
    innermost cache stride, and that every tensor is on one device."""
    import torch
    for name, t in (("q", q), ("k_cache", k_cache), ("out", out)) + ((("v_cache", v_cache),) if v_cache is not None else ()):
        _require(t.dtype == torch.bfloat16, f"{name} must be bfloat16, not {t.dtype}")
    for name, t in (("block_table", block_table), ("seq_lens", seq_lens), ("query_start_loc", query_start_loc)):
        _require(t.dtype == torch.int32, f"{name} must be int32, not {t.dtype}")
    _require(lse is None or lse.dtype == torch.float32, "lse must be float32")
    for name, t in (("q", q), ("out", out), ("seq_lens", seq_lens), ("query_start_loc", query_start_loc)) + \
            ((("lse", lse),) if lse is not None else ()):
        _require(t.is_contiguous(), f"{name} must be contiguous")
    _require(block_table.dim() == 2 and block_table.stride(1) == 1, "block_table must be 2-D with unit column stride")
    for name, t in (("k_cache", k_cache),) + ((("v_cache", v_cache),) if v_cache is not None else ()):
        _require(t.dim() == 4 and t.stride(3) == 1, f"{name} must be [pages, P, Hkv, d] with a unit innermost stride")
    devs = {t.device for t in (q, k_cache, block_table, seq_lens, query_start_loc, out)
            if t is not None}
    _require(len(devs) == 1, f"tensors on several devices: {devs}")
    a = Args()
    a.q = q.data_ptr()
    a.k_cache = k_cache.data_ptr()
    a.v_cache = v_cache.data_ptr() if v_cache is not None else None
    ks = k_cache.stride()
    a.k_stride = (ctypes.c_int64 * 3)(ks[0], ks[1], ks[2])
    vsrc = v_cache if v_cache is not None else k_cache
    vs = vsrc.stride()
    a.v_stride = (ctypes.c_int64 * 3)(vs[0], vs[1], vs[2])
    a.num_pages = k_cache.shape[0]
    a.block_table = block_table.data_ptr()
    a.block_table_stride = block_table.stride(0)
    a.seq_lens = seq_lens.data_ptr()
    a.query_start_loc = query_start_loc.data_ptr()
    a.out = out.data_ptr()
    a.lse = lse.data_ptr() if lse is not None else None
    if d_plan is not None:
        a.d_plan = d_plan.data_ptr()
        a.d_plan_bytes = d_plan.numel() * d_plan.element_size()
    if workspace is not None:
        a.workspace = workspace.data_ptr()
        a.workspace_bytes = workspace.numel() * workspace.element_size()
    return a


def flex_attn_plan_upload(plan: Plan, d_plan, stream=None):
    s = stream if stream is not None else current_stream()
    check(lib().flex_attn_plan_upload(plan.handle, ctypes.c_void_p(d_plan.data_ptr()),
                                      d_plan.numel() * d_plan.element_size(), s), "flex_attn_plan_upload")


class _PlanCopy:
    """A plan's copy to the device, which is queued on the stream that is current here:
    a run on another stream waits for it, the first time."""

    def __init__(self, device):
        import torch
        self.device, self.event = device, None
        if device.type != "cuda" or torch.cuda.is_current_stream_capturing():   # (in a graph: its own order)
            return
        s = torch.cuda.current_stream(device)
        self.event, self.behind = s.record_event(), {s.cuda_stream}

    def order(self, stream):
        import torch
        if self.event is None:
            return
        handle = getattr(stream, "value", stream) or 0
        if handle in self.behind:
            return
        s = torch.cuda.ExternalStream(handle, device=self.device)
        with torch.cuda.stream(s):
            if torch.cuda.is_current_stream_capturing():   # a capture may not wait for what is outside of it
                return
        s.wait_event(self.event)
        self.behind.add(handle)


def _behind_plan_copy(args, stream):
    copy = getattr(args, "plan_copy", None)
    if copy is not None:
        copy.order(stream)
    return stream


def flex_attn_decode(plan: Plan, args: Args, stream=None):
    s = _behind_plan_copy(args, stream if stream is not None else current_stream())
    check(lib().flex_attn_decode(plan.handle, ctypes.byref(args), s), "flex_attn_decode")


def flex_attn_prefill(plan: Plan, args: Args, stream=None):
    s = _behind_plan_copy(args, stream if stream is not None else current_stream())
    check(lib().flex_attn_prefill(plan.handle, ctypes.byref(args), s), "flex_attn_prefill")


def flex_attn_mixed(plan: Plan, args: Args, mode: int, stream=None, corun: "Corun" = None):
    s = _behind_plan_copy(args, stream if stream is not None else current_stream())
    check(lib().flex_attn_mixed(plan.handle, ctypes.byref(args), mode, s,
                                corun.handle if corun is not None else None), "flex_attn_mixed")


def flex_attn_validate_host(plan: Plan, block_table, num_pages: int, seq_lens, query_start_loc):
    """Host-side check of a run's metadata against the plan (torch CPU int32 tensors or int lists).
    Raises FlexAttnError (FLEX_ERR_INVALID_ARG) naming the first violation."""
    import torch
    bt = torch.as_tensor(block_table, dtype=torch.int32).contiguous()
    if bt.dim() != 2:
        raise ValueError("block_table must be 2-D")
    ptr = ctypes.cast(bt.data_ptr(), ctypes.POINTER(ctypes.c_int32))
    check(lib().flex_attn_validate_host(plan.handle, ptr, bt.stride(0), int(num_pages), _i32_array(seq_lens),
                                        _i32_array(query_start_loc)), "flex_attn_validate_host")


def set_debug(level: int) -> int:
    """Debug mode of the run calls (device check before launch); returns the previous level."""
    r = lib().flex_attn_set_debug(int(level))
    if r < 0:
        check(r, "flex_attn_set_debug")
    return r


def flex_attn_mixed_static(plan: Plan, args: Args, mode: int, stream=None, corun: "Corun" = None):
    """flex_attn_mixed with the split-K partials in the library's fixed scratch (allocates nothing)."""
    s = _behind_plan_copy(args, stream if stream is not None else current_stream())
    check(lib().flex_attn_mixed_static(plan.handle, ctypes.byref(args), mode, s,
                                       corun.handle if corun is not None else None), "flex_attn_mixed_static")


def static_scratch_bytes() -> int:
    return int(lib().flex_attn_static_scratch_bytes())


def flex_attn_debug_gather(plan: Plan, args: Args, seq: int, seq_len: int, k_out, v_out=None, stream=None):
    s = stream if stream is not None else current_stream()
    check(lib().flex_attn_debug_gather(plan.handle, ctypes.byref(args), seq, seq_len, _ptr(k_out),
                                       _ptr(v_out), s), "flex_attn_debug_gather")


def flex_attn_workspace_init(workspace, stream=None):
    s = stream if stream is not None else current_stream()
    check(lib().flex_attn_workspace_init(ctypes.c_void_p(workspace.data_ptr()),
                                         workspace.numel() * workspace.element_size(), s),
          "flex_attn_workspace_init")


def make_append_args(k_new, v_new, slot_mapping, k_cache, v_cache, bad_count=None) -> AppendArgs:
    """AppendArgs from device tensors: k_new [n, Hkv, d_qk] / v_new [n, Hkv, d_v] with
    contiguous rows, slot_mapping int32 [n], caches [pages, P, Hkv, d]."""
    a = AppendArgs()
    a.k_new = k_new.data_ptr()
    a.k_new_stride = k_new.stride(0)
    if v_new is not None:
        a.v_new = v_new.data_ptr()
        a.v_new_stride = v_new.stride(0)
    a.slot_mapping = slot_mapping.data_ptr()
    a.n_tokens = slot_mapping.numel()
    a.k_cache = k_cache.data_ptr()
    ks = k_cache.stride()
    a.k_stride = (ctypes.c_int64 * 3)(ks[0], ks[1], ks[2])
    vsrc = v_cache if v_cache is not None else k_cache
    a.v_cache = v_cache.data_ptr() if v_cache is not None else None
    vs = vsrc.stride()
    a.v_stride = (ctypes.c_int64 * 3)(vs[0], vs[1], vs[2])
    a.num_pages = k_cache.shape[0]
    a.bad_count = bad_count.data_ptr() if bad_count is not None else None
    return a


def flex_attn_kv_append(shape: Shape, args: AppendArgs, stream=None):
    s = stream if stream is not None else current_stream()
    check(lib().flex_attn_kv_append(ctypes.byref(shape), ctypes.byref(args), s), "flex_attn_kv_append")


def _one_device(tensors):
    """The device of the tensors given (None skipped); ValueError if there are several."""
    devs = {t.device for t in tensors if t is not None}
    _require(len(devs) == 1, f"tensors on several devices: {devs}")
    return devs.pop()


def _run(what, args, stream, *call, last=()):
    """Calls lib().<what>(*call, stream, *last) on the device of args' tensors, on its
    current stream unless one is given. ValueError for tensors that are not on a GPU."""
    import torch
    dev = args.device
    if dev.type != "cuda":
        raise ValueError(f"{what} needs GPU tensors, not {dev}")
    if dev.index == torch.cuda.current_device():
        s = _behind_plan_copy(args, stream if stream is not None else current_stream())
        st = getattr(lib(), what)(*call, s, *last)
    else:
        with torch.cuda.device(dev):
            s = _behind_plan_copy(args, stream if stream is not None else current_stream())
            st = getattr(lib(), what)(*call, s, *last)
    if st != FLEX_OK:
        check(st, what)


def _rows(name, t, heads, dim, dtype=None):
    """Checks a [tokens, heads, dim] tensor whose rows have no gaps; returns the token stride."""
    import torch
    _require(t.dtype == (dtype or torch.bfloat16), f"{name} must be {dtype or torch.bfloat16}, not {t.dtype}")
    _require(t.dim() == 3 and tuple(t.shape[1:]) == (heads, dim), f"{name} must be [tokens, {heads}, {dim}]")
    _require(t.shape[0] == 0 or ((dim == 1 or t.stride(2) == 1) and (heads == 1 or t.stride(1) == dim)),
             f"{name} must have contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else heads * dim


def _cache(name, t, heads, dtype):
    _require(t.dtype == dtype, f"{name} must be {dtype}, not {t.dtype}")
    _require(t.dim() == 4 and t.shape[2] == heads and t.stride(3) == 1,
             f"{name} must be [pages, P, {heads}, d] with a unit innermost stride")
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


def _index(name, t, shape=None):
    import torch
    _require(t.dtype == torch.int32, f"{name} must be int32, not {t.dtype}")
    _require(t.is_contiguous(), f"{name} must be contiguous")
    _require(shape is None or tuple(t.shape) == tuple(shape), f"{name} must be {list(shape or ())}")
    return t.data_ptr()


def rope_table(max_position: int, rot_dim: int, base: float = 10000.0, device="cuda"):
    """fp32 [max_position, rot_dim] for make_rope: cosines, then sines, of the
    angles p * base^(-2 i / rot_dim), worked out in 64 bits (in 32, the angles
    of far positions are off by more than the table's rounding)."""
    import torch
    i = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
    angle = torch.arange(max_position, dtype=torch.float64, device=device)[:, None] * float(base) ** (-2.0 * i / rot_dim)
    return torch.cat([torch.cos(angle), torch.sin(angle)], 1).float()


def make_rope(cos_sin, positions=None, rot_begin: int = 0, neighbours: bool = False, sections=None,
              dealt: bool = False) -> Rope:
    """Rope from device tensors: cos_sin fp32 [max_position, rot_dim] (rope_table),
    positions int32 [tokens] or [axes, tokens] (rows may be apart), or None for
    flex_attn_kv8_append with one axis. sections: pairs of each axis, given
    when there is more than one. (This one, like the arguments of the calls that
    rotate or use an 8-bit cache, keeps its tensors.)"""
    import torch
    _require(cos_sin.dtype == torch.float32, f"cos_sin must be float32, not {cos_sin.dtype}")
    _require(cos_sin.dim() == 2 and cos_sin.is_contiguous(), "cos_sin must be [max_position, rot_dim], contiguous")
    r = Rope()
    r.cos_sin = cos_sin.data_ptr()
    r.max_position, r.rot_dim = cos_sin.shape
    r.rot_begin, r.neighbours, r.dealt, r.n_axes = rot_begin, int(bool(neighbours)), int(bool(dealt)), 1
    r.n_positions = None
    if positions is not None:
        _require(positions.dtype == torch.int32, f"positions must be int32, not {positions.dtype}")
        p = positions[None] if positions.dim() == 1 else positions
        _require(p.dim() == 2 and (p.shape[1] <= 1 or p.stride(1) == 1), "positions must be [axes, tokens] with unit column stride")
        r.positions, r.n_axes, r.n_positions = p.data_ptr(), p.shape[0], p.shape[1]
        r.positions_stride = p.stride(0) if p.shape[0] > 1 else p.shape[1]
    axes = list(sections) if sections is not None else []
    _require(len(axes) == (r.n_axes if r.n_axes > 1 else len(axes)) and len(axes) <= FLEX_ROPE_MAX_AXES,
             f"sections must name the pairs of {r.n_axes} axes")
    for a, n in enumerate(axes):
        r.sections[a] = n
    r.device = _one_device([cos_sin, positions])
    r.tensors = (cos_sin, positions)
    return r


def _check_rope(rope, args, n_tokens):
    if rope.device != args.device:
        raise ValueError(f"rope on {rope.device}, tensors on {args.device}")
    if rope.n_positions is not None and rope.n_positions < n_tokens:
        raise ValueError(f"{rope.n_positions} positions for {n_tokens} tokens")


def make_rope_append_args(q, q_out, k_new, v_new, slot_mapping, k_cache, v_cache, bad_count=None) -> RopeAppendArgs:
    """RopeAppendArgs from device tensors: q [n, Hq, d_qk] with contiguous rows,
    q_out [n, Hq, d_qk] contiguous (q itself to turn it in place), the rest as
    for make_append_args (v_new and v_cache None when values alias keys)."""
    import torch
    n, (Hq, dk), Hkv = q.shape[0], q.shape[1:], k_cache.shape[2]
    a = RopeAppendArgs()
    a.q, a.q_stride, a.q_out = q.data_ptr(), _rows("q", q, Hq, dk), q_out.data_ptr()
    _require(q_out.shape == q.shape and q_out.dtype == torch.bfloat16 and q_out.is_contiguous(),
             "q_out must be like q, contiguous")
    _require((v_new is None) == (v_cache is None), "v_new and v_cache are given together")
    a.kv.k_new, a.kv.k_new_stride = k_new.data_ptr(), _rows("k_new", k_new, Hkv, dk)
    a.kv.k_stride, a.kv.k_cache = _cache("k_cache", k_cache, Hkv, torch.bfloat16), k_cache.data_ptr()
    a.kv.v_stride, a.kv.num_pages, a.kv.n_tokens = a.kv.k_stride, k_cache.shape[0], n
    if v_new is not None:
        a.kv.v_new, a.kv.v_new_stride = v_new.data_ptr(), _rows("v_new", v_new, Hkv, v_cache.shape[3])
        a.kv.v_stride, a.kv.v_cache = _cache("v_cache", v_cache, Hkv, torch.bfloat16), v_cache.data_ptr()
        _require(v_cache.shape[:2] == k_cache.shape[:2], "k_cache and v_cache must have the same pages")
    a.kv.slot_mapping = _index("slot_mapping", slot_mapping, (n,))
    _require(k_new.shape[0] == n and (v_new is None or v_new.shape[0] == n), "q, k_new and v_new must have the same tokens")
    if bad_count is not None:
        a.kv.bad_count = _index("bad_count", bad_count)
    a.tensors = (q, q_out, k_new, v_new, slot_mapping, k_cache, v_cache, bad_count)
    a.device = _one_device(a.tensors)
    a.sizes = (Hq, Hkv, dk, None if v_new is None else v_cache.shape[3], k_cache.shape[1])
    return a


def _check_sizes(shape, args):
    """args.sizes: query heads (None: no queries), KV heads, key and value width (None: aliased), page size."""
    hq, *rest = args.sizes
    want = [shape.num_kv_heads, shape.head_dim_qk, None if shape.v_aliases_k else shape.head_dim_v, shape.page_size]
    if rest != want or (hq is not None and hq != shape.num_q_heads):
        raise ValueError(f"tensors for {args.sizes}, shape {(shape.num_q_heads, *want)}")


def flex_attn_rope_append(shape: Shape, rope: Rope, args: RopeAppendArgs, stream=None):
    _check_sizes(shape, args)
    _check_rope(rope, args, args.kv.n_tokens)
    _run("flex_attn_rope_append", args, stream, ctypes.byref(shape), ctypes.byref(rope), ctypes.byref(args))


def make_kv8_cache(num_pages: int, page_size: int, num_kv_heads: int, head_dim: int, device="cuda"):
    """(k_cache, v_cache, kv_scales) of an empty 8-bit cache: e4m3 codes
    [pages, P, Hkv, d] and e8m0 scales [pages, P / 16, Hkv, 2], all zero bytes."""
    import torch
    k, v = (torch.zeros((num_pages, page_size, num_kv_heads, head_dim), dtype=torch.uint8, device=device) for _ in "kv")
    s = torch.zeros((num_pages, page_size // 16, num_kv_heads, 2), dtype=torch.uint8, device=device)
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu)


def _check_kv8(k_cache, v_cache, kv_scales):
    """Checks an 8-bit cache; returns (k strides, v strides, scale page stride)."""
    import torch
    pages, P, heads = k_cache.shape[:3]
    ks = _cache("k_cache", k_cache, heads, torch.float8_e4m3fn)
    vs = _cache("v_cache", v_cache, heads, torch.float8_e4m3fn)
    _require(v_cache.shape == k_cache.shape, "k_cache and v_cache must have the same shape")
    _require(kv_scales.dtype == torch.float8_e8m0fnu, f"kv_scales must be float8_e8m0fnu, not {kv_scales.dtype}")
    _require(P % 16 == 0 and tuple(kv_scales.shape) == (pages, P // 16, heads, 2),
             f"kv_scales must be [{pages}, {P} / 16, {heads}, 2]")
    _require(pages == 0 or kv_scales[0].is_contiguous(), "kv_scales must be contiguous within a page")
    return ks, vs, kv_scales.stride(0) if pages > 1 else P // 16 * heads * 2


def make_kv8_append_args(k_new, v_new, block_table, seq_lens, query_start_loc, k_cache, v_cache, kv_scales, q=None,
                         q_out=None, bad_count=None) -> Kv8AppendArgs:
    """Kv8AppendArgs from device tensors: k_new / v_new [n, Hkv, d] with
    contiguous rows, the batch's block_table, seq_lens and query_start_loc as
    the attention takes them, an 8-bit cache (make_kv8_cache), and q
    [n, Hq, d] with q_out (contiguous, may be q) when a rotation is applied."""
    import torch
    n, B = k_new.shape[0], seq_lens.numel()
    heads, d = k_cache.shape[2:]
    a = Kv8AppendArgs()
    a.k_stride, a.v_stride, a.scale_page_stride = _check_kv8(k_cache, v_cache, kv_scales)
    a.k_new, a.k_new_stride = k_new.data_ptr(), _rows("k_new", k_new, heads, d)
    a.v_new, a.v_new_stride = v_new.data_ptr(), _rows("v_new", v_new, heads, d)
    _require(v_new.shape[0] == n, "k_new and v_new must have the same tokens")
    _require((q is None) == (q_out is None), "q and q_out are given together")
    Hq = None
    if q is not None:
        Hq = q.shape[1]
        a.q, a.q_stride, a.q_out = q.data_ptr(), _rows("q", q, Hq, d), q_out.data_ptr()
        _require(q_out.shape == q.shape and q_out.dtype == torch.bfloat16 and q_out.is_contiguous(),
                 "q_out must be like q, contiguous")
        _require(q.shape[0] == n, "q and k_new must have the same tokens")
    a.n_tokens, a.num_seqs, a.num_pages = n, B, k_cache.shape[0]
    _require(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.stride(1) == 1 and
             block_table.shape[0] == B, "block_table must be int32 [sequences, pages] with unit column stride")
    a.block_table = block_table.data_ptr()
    a.block_table_stride = block_table.stride(0) if B > 1 else block_table.shape[1]
    a.seq_lens, a.query_start_loc = _index("seq_lens", seq_lens, (B,)), _index("query_start_loc", query_start_loc, (B + 1,))
    a.k_cache, a.v_cache, a.kv_scales = k_cache.data_ptr(), v_cache.data_ptr(), kv_scales.data_ptr()
    if bad_count is not None:
        a.bad_count = _index("bad_count", bad_count)
    a.tensors = (k_new, v_new, block_table, seq_lens, query_start_loc, k_cache, v_cache, kv_scales, q, q_out, bad_count)
    a.device = _one_device(a.tensors)
    a.sizes = (Hq, heads, d, d, k_cache.shape[1])
    return a


def flex_attn_kv8_append(shape: Shape, rope: Optional[Rope], args: Kv8AppendArgs, stream=None):
    _check_sizes(shape, args)
    if rope is not None:
        _check_rope(rope, args, args.n_tokens)
    _run("flex_attn_kv8_append", args, stream, ctypes.byref(shape), ctypes.byref(rope) if rope is not None else None,
         ctypes.byref(args))


def make_kv8_args(q, k_cache, v_cache, kv_scales, block_table, seq_lens, query_start_loc, out, lse=None, d_plan=None,
                  workspace=None) -> Kv8Args:
    """Kv8Args from device tensors: as make_args, over an 8-bit cache (make_kv8_cache)."""
    import torch
    a = Kv8Args()
    ks, vs, a.scale_page_stride = _check_kv8(k_cache, v_cache, kv_scales)
    # the rest is checked as for a bf16 cache, with q standing in for it
    a.attn = make_args(q, q[:0, None], q[:0, None], block_table, seq_lens, query_start_loc, out, lse, d_plan, workspace)
    a.attn.k_cache, a.attn.v_cache, a.attn.k_stride, a.attn.v_stride = k_cache.data_ptr(), v_cache.data_ptr(), ks, vs
    a.attn.num_pages = k_cache.shape[0]
    a.kv_scales = kv_scales.data_ptr()
    a.tensors = (q, k_cache, v_cache, kv_scales, block_table, seq_lens, query_start_loc, out, lse, d_plan, workspace)
    a.device = _one_device(a.tensors)
    _require(q.dim() == 3, "q must be [tokens, Hq, d]")
    _require(out.shape[:2] == q.shape[:2] and out.shape[2:] == v_cache.shape[3:], "out must be [tokens, Hq, d]")
    _require(lse is None or lse.shape == q.shape[:2], "lse must be [tokens, Hq]")
    a.sizes = (q.shape[1], k_cache.shape[2], q.shape[2], v_cache.shape[3], k_cache.shape[1])
    a.batch = (seq_lens.numel(), q.shape[0])
    _require(block_table.shape[0] == a.batch[0] and query_start_loc.numel() == a.batch[0] + 1,
             "block_table, seq_lens and query_start_loc must be of as many sequences")
    return a


def _check_plan(plan, args):
    _check_sizes(plan.shape, args)
    if args.batch[0] != plan.batch[0] or args.batch[1] < plan.batch[1]:
        raise ValueError(f"tensors of {args.batch[0]} sequences and {args.batch[1]} tokens, a plan for {plan.batch[0]} and {plan.batch[1]}")


def flex_attn_decode_kv8(plan: Plan, args: Kv8Args, stream=None):
    _check_plan(plan, args)
    _run("flex_attn_decode_kv8", args, stream, plan.handle, ctypes.byref(args))


def flex_attn_prefill_kv8(plan: Plan, args: Kv8Args, stream=None):
    _check_plan(plan, args)
    _run("flex_attn_prefill_kv8", args, stream, plan.handle, ctypes.byref(args))


def flex_attn_mixed_kv8(plan: Plan, args: Kv8Args, mode: int, stream=None, corun: "Corun" = None):
    _check_plan(plan, args)
    _run("flex_attn_mixed_kv8", args, stream, plan.handle, ctypes.byref(args), mode,
         last=(corun.handle if corun is not None else None,))


class Controller:
    """The online co-location controller (flex_ctl_*): observe steps, decide splits."""

    def __init__(self, **opts):
        o = CtlOpts()
        for k, v in opts.items():
            setattr(o, k, v)
        h = ctypes.c_void_p()
        check(lib().flex_ctl_create(ctypes.byref(o), ctypes.byref(h)), "flex_ctl_create")
        self.handle = h
        self.K = (o.cus_total or 256) // (o.granule or 64)

    def close(self):
        if self.handle:
            lib().flex_ctl_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_profile(self, cus, decode_gbps, prefill_tflops):
        n = len(cus)
        check(lib().flex_ctl_set_profile(self.handle, n, (ctypes.c_int32 * n)(*cus),
                                         (ctypes.c_double * n)(*decode_gbps), (ctypes.c_double * n)(*prefill_tflops)),
              "flex_ctl_set_profile")

    def observe(self, cus_decode, decode_bytes, prefill_flops, decode_ms, prefill_ms, fused=False, step_ms=0.0):
        ob = CtlObservation(cus_decode, decode_bytes, prefill_flops, decode_ms, prefill_ms, 1 if fused else 0, step_ms)
        check(lib().flex_ctl_observe(self.handle, ctypes.byref(ob)), "flex_ctl_observe")

    def decide(self, decode_bytes, prefill_flops, pending_prefill_tokens=0, pending_decode_seqs=0,
               active_decode_seqs=1, fused_available=False, decode_tail=False) -> dict:
        sg = CtlSignals(decode_bytes, prefill_flops, pending_prefill_tokens, pending_decode_seqs, active_decode_seqs,
                        1 if fused_available else 0, 1 if decode_tail else 0)
        d = CtlDecision()
        check(lib().flex_ctl_decide(self.handle, ctypes.byref(sg), ctypes.byref(d)), "flex_ctl_decide")
        return {"mode": d.mode, "cus_decode": d.cus_decode, "cus_prefill": d.cus_prefill, "reason": d.reason,
                "predicted_us": d.predicted_us}

    def estimates(self):
        dg, pt = (ctypes.c_double * self.K)(), (ctypes.c_double * self.K)()
        check(lib().flex_ctl_estimates(self.handle, dg, pt, self.K), "flex_ctl_estimates")
        return list(dg), list(pt)


class TimeSlice:
    """The time-slice scheduler (flex_ts_*): one phase per step, decode's share
    of the device time held near decode_share."""

    def __init__(self, decode_share=0.5, decay=1.0):
        h = ctypes.c_void_p()
        check(lib().flex_ts_create(ctypes.byref(TsOpts(decode_share, decay)), ctypes.byref(h)), "flex_ts_create")
        self.handle = h

    def close(self):
        if self.handle:
            lib().flex_ts_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def next(self, decode_ready: bool, prefill_ready: bool) -> int:
        ph = ctypes.c_int32()
        check(lib().flex_ts_next(self.handle, int(bool(decode_ready)), int(bool(prefill_ready)), ctypes.byref(ph)),
              "flex_ts_next")
        return ph.value

    def observe(self, phase: int, ms: float):
        check(lib().flex_ts_observe(self.handle, int(phase), float(ms)), "flex_ts_observe")

    def totals(self):
        d, p = ctypes.c_double(), ctypes.c_double()
        check(lib().flex_ts_totals(self.handle, ctypes.byref(d), ctypes.byref(p)), "flex_ts_totals")
        return d.value, p.value


class Corun:
    """Owning wrapper of a co-run stream pair (two CU-masked streams)."""

    def __init__(self, cus_prefill: int, cus_decode: int):
        h = ctypes.c_void_p()
        check(lib().flex_attn_corun_create(cus_prefill, cus_decode, ctypes.byref(h)), "flex_attn_corun_create")
        self.handle = h
        self.cus_prefill = cus_prefill
        self.cus_decode = cus_decode

    def streams(self):
        p, d = ctypes.c_void_p(), ctypes.c_void_p()
        check(lib().flex_attn_corun_streams(self.handle, ctypes.byref(p), ctypes.byref(d)),
              "flex_attn_corun_streams")
        return p.value, d.value

    def set_timing(self, enable: bool = True):
        check(lib().flex_attn_corun_set_timing(self.handle, 1 if enable else 0), "flex_attn_corun_set_timing")

    def timing_read(self):
        """(prefill_ms, decode_ms) lists of the recorded steps, oldest first (waits for them)."""
        n = FLEX_TIMING_RING
        pre = (ctypes.c_float * n)()
        dec = (ctypes.c_float * n)()
        cnt = ctypes.c_int32()
        check(lib().flex_attn_corun_timing_read(self.handle, pre, dec, n, ctypes.byref(cnt)),
              "flex_attn_corun_timing_read")
        return list(pre[:cnt.value]), list(dec[:cnt.value])

    def close(self):
        if self.handle and self.handle.value:
            lib().flex_attn_corun_destroy(self.handle)
            self.handle = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class PagedAttention:
    """One batch's plan, its device copy and its workspace (torch-allocated).

    ``inputs`` holds the device tensors: q, k_cache, v_cache (or None when V
    aliases K), block_table, seq_lens, query_start_loc (int32). ``run`` calls
    the library on the current torch stream. The plan is copied to the device
    on its stream that is current at construction; a run on another stream
    with arguments made here waits for the copy (but in a capture, which cannot:
    there it has to be over).
    """

    def __init__(self, shape: Shape, opts: Optional[PlanOpts], h_query_start_loc, h_seq_lens,
                 max_pages_per_seq: int, device="cuda"):
        import torch
        self.shape = shape
        self.plan = flex_attn_plan(shape, opts, h_query_start_loc, h_seq_lens, max_pages_per_seq)
        info = self.plan.info
        self.d_plan = torch.empty(max(256, info["device_plan_bytes"]), dtype=torch.uint8, device=device)
        self.workspace = torch.empty(max(256, info["workspace_bytes"]), dtype=torch.uint8, device=device)
        with torch.cuda.device(self.d_plan.device):
            flex_attn_plan_upload(self.plan, self.d_plan)
            self.plan_copy = _PlanCopy(self.d_plan.device)

    def args(self, q, k_cache, v_cache, block_table, seq_lens, query_start_loc, out, lse=None) -> Args:
        a = make_args(q, k_cache, v_cache, block_table, seq_lens, query_start_loc, out, lse,
                      self.d_plan, self.workspace)
        a.plan_copy = self.plan_copy
        return a

    def kv8_args(self, q, k_cache, v_cache, kv_scales, block_table, seq_lens, query_start_loc, out, lse=None) -> Kv8Args:
        """Arguments of the calls over an 8-bit cache (a plan made with kv_bits=8)."""
        a = make_kv8_args(q, k_cache, v_cache, kv_scales, block_table, seq_lens, query_start_loc, out, lse,
                          self.d_plan, self.workspace)
        a.plan_copy = self.plan_copy
        return a

    def alloc_out(self, q, with_lse=False):
        import torch
        T, Hq = q.shape[0], q.shape[1]
        out = torch.empty((T, Hq, self.shape.head_dim_v), dtype=torch.bfloat16, device=q.device)
        lse = torch.empty((T, Hq), dtype=torch.float32, device=q.device) if with_lse else None
        return out, lse
