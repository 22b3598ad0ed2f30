"""ctypes binding of libfcp.so: same names as the C ABI in include/fcp.h, argument marshalling only.

Every step of the path runs inside the library's kernels; PyTorch is used by callers for device
memory and streams.  There is no fallback: if the shared library is missing, `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfcp.so")

FCP_OK = 0
FCP_ERR_INVALID_ARG, FCP_ERR_INFEASIBLE, FCP_ERR_UNSUPPORTED, FCP_ERR_WORKSPACE = -1, -2, -3, -4
FCP_ERR_CUDA, FCP_ERR_TIMEOUT, FCP_ERR_NOT_UPLOADED, FCP_ERR_NO_MEMORY = -5, -6, -7, -8
FCP_MAX_DEGREE = 64

TABLES = dict(cu_seqlens=0, chunk_offset=1, chunk_bounds=2, pairs=3, items=4, slot_offset=5, slot_rows=6,
              fwd_units=7, bwd_units=8, bwd_qranges=9, merge_units=10, bwd_work=11, fused_units=12, row_limit=13,
              first_query=14, span_pairs=15, fwd_groups=16, fused_groups=17, bwd_groups=18)
_TABLE_WIDTH = dict(pairs=6, items=8, fwd_units=16, bwd_units=8, bwd_qranges=4, merge_units=4, fused_units=16,
                    span_pairs=5, fwd_groups=4, fused_groups=4, bwd_groups=4)
INFO = dict(T=0, R=1, n_pairs=2, n_items=3, n_fwd_units=4, n_bwd_units=5, n_merge_units=6, B=7, n_merge_multi=8,
            n_fused_units=9, fused_split=10)

EXPORTS = ["fcp_plan_strategy", "fcp_plan_blocks", "fcp_plan_blocks_spans", "fcp_span_mask_efficiency", "fcp_plan_get", "fcp_plan_info", "fcp_plan_workspace_bytes",
           "fcp_plan_bwd_scratch_bytes", "fcp_plan_upload", "fcp_release_cached", "fcp_plan_destroy", "fcp_attn_fwd", "fcp_attn_fwd_merged",
           "fcp_attn_fwd_fused", "fcp_lse_merge", "fcp_attn_bwd", "fcp_attn_bwd_heads",
           "fcp_host_workspace_bytes", "fcp_attn_fwd_bwd_host", "fcp_last_device_status", "fcp_plan_set_profiling",
           "fcp_plan_kernel_ms", "fcp_noalloc_bytes_needed", "fcp_attn_bwd_noalloc", "fcp_noalloc_device_status",
           "fcp_rope_init", "fcp_rope_fwd", "fcp_rope_bwd", "fcp_cache_create", "fcp_cache_destroy",
           "fcp_cache_device_status", "fcp_cache_append", "fcp_cache_attn_workspace_bytes", "fcp_cache_attn", "fcp_cache_evict",
           "fcp_selftest_bounded_wait", "fcp_status_string",
           "fcp_last_error_message"]


class FcpParams(C.Structure):
    _fields_ = [("hq", C.c_int32), ("hkv", C.c_int32), ("head_dim", C.c_int32), ("scale", C.c_float)]


class FcpCostCoeffs(C.Structure):
    _fields_ = [("alpha1", C.c_double), ("alpha2", C.c_double), ("alpha3", C.c_double), ("beta1", C.c_double),
                ("beta2", C.c_double), ("v", C.c_double), ("eta", C.POINTER(C.c_double))]


class FcpRopeConfig(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("base", C.c_double), ("factor", C.c_double), ("original_length", C.c_double), ("low", C.c_double),
                ("high", C.c_double), ("magnitude", C.c_double)]


class FcpRopeTable(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("layout", C.c_int32), ("magnitude", C.c_float),
                ("turn", C.c_uint64 * 64)]


class FcpCacheConfig(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("weight", C.c_void_p), ("status", C.c_void_p), ("n_pages", C.c_int32), ("page_tokens", C.c_int32),
                ("hkv", C.c_int32), ("head_dim", C.c_int32), ("kind", C.c_int32)]


class FcpCacheBatch(C.Structure):
    _fields_ = [("B", C.c_int32), ("rows", C.c_int32), ("max_new", C.c_int32), ("table_width", C.c_int32),
                ("page_table", C.c_void_p), ("length", C.c_void_p), ("row_offset", C.c_void_p)]


class FcpError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{status_string(status)}: {message}")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    """Loads libfcp.so (built by paper_2602_21788_b200/build.py).  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(f"{LIB_PATH} is missing: run `python -m paper_2602_21788_b200.build` (needs nvcc)")
    L = C.CDLL(LIB_PATH)
    i32p, i64p, f32p, f64p, vp = (C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_float),
                                  C.POINTER(C.c_double), C.c_void_p)
    L.fcp_plan_strategy.argtypes = [i32p, C.c_int32, C.c_int32, C.c_double, C.c_double, C.c_double,
                                    C.POINTER(FcpCostCoeffs), i32p, i32p, i32p, f64p]
    L.fcp_plan_blocks.argtypes = [i32p, i32p, C.c_int32, C.POINTER(FcpParams), C.POINTER(vp)]
    L.fcp_plan_blocks_spans.argtypes = [i32p, i32p, C.c_int32, i32p, i32p, C.POINTER(FcpParams), C.POINTER(vp)]
    L.fcp_span_mask_efficiency.argtypes = [C.c_int32, i32p, C.c_int32, f64p]
    L.fcp_plan_get.argtypes = [vp, C.c_int32, C.POINTER(i32p), i64p]
    L.fcp_plan_info.argtypes = [vp, C.c_int32, i64p]
    L.fcp_plan_workspace_bytes.argtypes = [vp, C.c_int32, i64p, i64p, i64p]
    L.fcp_plan_upload.argtypes = [vp, vp]
    L.fcp_plan_destroy.argtypes = [vp]
    L.fcp_release_cached.argtypes = []
    L.fcp_attn_fwd.argtypes = [vp, vp, vp, vp, C.c_int32, C.c_int32, vp, vp, vp]
    L.fcp_lse_merge.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp]
    L.fcp_attn_fwd_merged.argtypes = [vp, vp, vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp, vp]
    L.fcp_plan_set_profiling.argtypes = [vp, C.c_int32]
    L.fcp_plan_kernel_ms.argtypes = [vp, C.c_int32, i32p, f32p]
    L.fcp_attn_bwd.argtypes = [vp] * 11 + [C.c_int64, vp]
    L.fcp_attn_bwd_heads.argtypes = [vp] * 7 + [C.c_int32, C.c_int32] + [vp] * 4 + [C.c_int64, vp]
    L.fcp_attn_fwd_fused.argtypes = [vp, vp, vp, vp, C.c_int32, C.c_int32, vp, vp, vp, vp]
    L.fcp_plan_bwd_scratch_bytes.argtypes = [vp, C.c_int32, i64p]
    L.fcp_host_workspace_bytes.argtypes = [vp, i64p]
    L.fcp_attn_fwd_bwd_host.argtypes = [vp] * 11 + [C.c_int64, vp]
    L.fcp_last_device_status.argtypes = [vp, i32p]
    L.fcp_noalloc_bytes_needed.argtypes = [vp, i64p]
    L.fcp_attn_bwd_noalloc.argtypes = [vp] * 11
    L.fcp_noalloc_device_status.argtypes = [i32p]
    L.fcp_rope_init.argtypes = [C.POINTER(FcpRopeConfig), C.POINTER(FcpRopeTable)]
    for f in (L.fcp_rope_fwd, L.fcp_rope_bwd):
        f.argtypes = [C.POINTER(FcpRopeTable), C.c_int64, vp, C.c_int64, C.c_int32, vp, C.c_int64, C.c_int32, vp, C.c_int64, vp,
                      C.c_int64, vp, vp, vp, C.c_int32, vp]
    batch = C.POINTER(FcpCacheBatch)
    L.fcp_cache_create.argtypes = [C.POINTER(FcpCacheConfig), C.POINTER(vp)]
    L.fcp_cache_destroy.argtypes = [vp]
    L.fcp_cache_device_status.argtypes = [vp, i32p]
    L.fcp_cache_append.argtypes = [vp, batch, vp, C.c_int64, vp, C.c_int64, vp]
    L.fcp_cache_attn_workspace_bytes.argtypes = [vp, batch, C.c_int32, i64p]
    L.fcp_cache_attn.argtypes = [vp, batch, vp, C.c_int64, C.c_int32, C.c_float, vp, vp, C.c_int32, vp, C.c_int64, vp]
    L.fcp_cache_evict.argtypes = [vp, batch, C.c_int32, C.c_int32, C.c_int32, vp, C.c_int32, vp, vp, vp]
    L.fcp_selftest_bounded_wait.argtypes = [C.c_uint32, i32p, vp]
    L.fcp_status_string.argtypes = [C.c_int]
    L.fcp_status_string.restype = C.c_char_p
    L.fcp_last_error_message.restype = C.c_char_p
    for name in EXPORTS:
        if name not in ("fcp_status_string", "fcp_last_error_message"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().fcp_status_string(int(status)).decode()


def _check(rc: int):
    if rc != FCP_OK:
        raise FcpError(rc, lib().fcp_last_error_message().decode())


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(C.c_int32))


def _ptr(x):
    """Raw address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return C.c_void_p(x)
    if isinstance(x, np.ndarray):
        return C.c_void_p(x.ctypes.data)
    return C.c_void_p(x.data_ptr())


def fcp_plan_strategy(seqlens, N, E, M_token, M_ms, coeffs: dict, eta=None):
    """Returns dict(group_of, cp_degree, n_groups, makespan).  coeffs: alpha1..beta2, v."""
    sl, slp = _i32(seqlens)
    B = len(sl)
    eta_arr = None if eta is None else np.ascontiguousarray(eta, dtype=np.float64)
    cc = FcpCostCoeffs(coeffs["alpha1"], coeffs["alpha2"], coeffs["alpha3"], coeffs["beta1"], coeffs["beta2"],
                       coeffs["v"], None if eta_arr is None else eta_arr.ctypes.data_as(C.POINTER(C.c_double)))
    group_of = np.zeros(max(B, 1), dtype=np.int32)
    deg = np.zeros(max(B, 1), dtype=np.int32)
    ng = C.c_int32(0)
    mk = C.c_double(0.0)
    _check(lib().fcp_plan_strategy(slp, B, int(N), float(E), float(M_token), float(M_ms), C.byref(cc),
                                   group_of.ctypes.data_as(C.POINTER(C.c_int32)),
                                   deg.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(ng), C.byref(mk)))
    return dict(group_of=group_of[:B], cp_degree=deg[:B], n_groups=ng.value, makespan=mk.value)


class Plan:
    """Owns an fcp_plan handle."""

    def __init__(self, seqlens, cp_degrees, hq, hkv, head_dim, scale=0.0, spans=None):
        """spans: None, or one list of (begin, end) pairs per sequence (positions relative to its start)."""
        sl, slp = _i32(seqlens)
        dg, dgp = _i32(cp_degrees)
        if len(sl) != len(dg):
            raise ValueError("seqlens and cp_degrees differ in length")
        self.params = FcpParams(int(hq), int(hkv), int(head_dim), float(scale))
        self.handle = C.c_void_p()
        if spans is None:
            _check(lib().fcp_plan_blocks(slp, dgp, len(sl), C.byref(self.params), C.byref(self.handle)))
        else:
            if len(spans) != len(sl):
                raise ValueError("spans needs one list per sequence")
            off = np.zeros(len(sl) + 1, dtype=np.int32)
            off[1:] = np.cumsum([len(x) for x in spans])
            flat = np.asarray([v for x in spans for ab in x for v in ab], dtype=np.int32)
            so, sop = _i32(off)
            fl, flp = _i32(flat if flat.size else np.zeros(2, dtype=np.int32))
            _check(lib().fcp_plan_blocks_spans(slp, dgp, len(sl), sop, flp, C.byref(self.params), C.byref(self.handle)))
        self.hq, self.hkv, self.head_dim = int(hq), int(hkv), int(head_dim)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value and _lib is not None:
            _lib.fcp_plan_destroy(h)
            self.handle = None

    def table(self, name: str) -> np.ndarray:
        p = C.POINTER(C.c_int32)()
        n = C.c_int64(0)
        _check(lib().fcp_plan_get(self.handle, TABLES[name], C.byref(p), C.byref(n)))
        arr = np.ctypeslib.as_array(p, shape=(n.value,)).copy() if n.value else np.zeros(0, dtype=np.int32)
        w = _TABLE_WIDTH.get(name)
        return arr.reshape(-1, w) if w else arr

    def info(self, name: str) -> int:
        v = C.c_int64(0)
        _check(lib().fcp_plan_info(self.handle, INFO[name], C.byref(v)))
        return v.value

    def workspace_bytes(self, heads_per_pass=None):
        a, b, c = C.c_int64(0), C.c_int64(0), C.c_int64(0)
        _check(lib().fcp_plan_workspace_bytes(self.handle, int(heads_per_pass or self.hq), C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def bwd_scratch_bytes(self, kv_head_count=None) -> int:
        v = C.c_int64(0)
        _check(lib().fcp_plan_bwd_scratch_bytes(self.handle, int(kv_head_count or self.hkv), C.byref(v)))
        return v.value

    def host_workspace_bytes(self) -> int:
        v = C.c_int64(0)
        _check(lib().fcp_host_workspace_bytes(self.handle, C.byref(v)))
        return v.value

    def upload(self, stream=0):
        _check(lib().fcp_plan_upload(self.handle, C.c_void_p(stream)))
        return self

    def set_profiling(self, enable: bool):
        _check(lib().fcp_plan_set_profiling(self.handle, 1 if enable else 0))

    def kernel_ms(self, kind: int):
        n = C.c_int32(0)
        ms = C.c_float(0.0)
        _check(lib().fcp_plan_kernel_ms(self.handle, int(kind), C.byref(n), C.byref(ms)))
        return n.value, ms.value

    def device_status(self):
        st = np.zeros(4, dtype=np.int32)
        _check(lib().fcp_last_device_status(self.handle, st.ctypes.data_as(C.POINTER(C.c_int32))))
        return st


def fcp_release_cached():
    """Frees the device blocks that destroyed plans left for later ones (current CUDA context)."""
    _check(lib().fcp_release_cached())


def fcp_plan_blocks(seqlens, cp_degrees, hq, hkv, head_dim, scale=0.0) -> Plan:
    return Plan(seqlens, cp_degrees, hq, hkv, head_dim, scale)


def fcp_plan_blocks_spans(seqlens, cp_degrees, spans, hq, hkv, head_dim, scale=0.0) -> Plan:
    return Plan(seqlens, cp_degrees, hq, hkv, head_dim, scale, spans=spans)


def fcp_span_mask_efficiency(length, spans) -> float:
    """eta_k of one sequence (Eq. 4): visible pairs over the causal count, minus 1."""
    flat = np.asarray([v for ab in spans for v in ab], dtype=np.int32)
    fl, flp = _i32(flat if flat.size else np.zeros(2, dtype=np.int32))
    eta = C.c_double(0.0)
    _check(lib().fcp_span_mask_efficiency(int(length), flp, len(spans), C.byref(eta)))
    return eta.value


def fcp_attn_fwd(plan: Plan, q, k, v, o_partial, lse_partial, head_begin=0, head_count=None, stream=0):
    hc = plan.hq - head_begin if head_count is None else head_count
    _check(lib().fcp_attn_fwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), int(head_begin), int(hc), _ptr(o_partial),
                              _ptr(lse_partial), C.c_void_p(stream)))


def fcp_attn_fwd_merged(plan: Plan, q, k, v, o_partial, lse_partial, o, lse, head_begin=0, head_count=None, stream=0):
    hc = plan.hq - head_begin if head_count is None else head_count
    _check(lib().fcp_attn_fwd_merged(plan.handle, _ptr(q), _ptr(k), _ptr(v), int(head_begin), int(hc), _ptr(o_partial),
                                     _ptr(lse_partial), _ptr(o), _ptr(lse), C.c_void_p(stream)))


def fcp_attn_fwd_fused(plan: Plan, q, k, v, o, lse, head_begin=0, head_count=None, stream=0, o_f32=None):
    hc = plan.hq - head_begin if head_count is None else head_count
    _check(lib().fcp_attn_fwd_fused(plan.handle, _ptr(q), _ptr(k), _ptr(v), int(head_begin), int(hc), _ptr(o), _ptr(o_f32),
                                    _ptr(lse), C.c_void_p(stream)))


def fcp_lse_merge(plan: Plan, o_partial, lse_partial, o, lse, head_begin=0, head_count=None, stream=0, o_f32=None):
    hc = plan.hq - head_begin if head_count is None else head_count
    _check(lib().fcp_lse_merge(plan.handle, _ptr(o_partial), _ptr(lse_partial), int(head_begin), int(hc), _ptr(o),
                               _ptr(o_f32), _ptr(lse), C.c_void_p(stream)))


def fcp_attn_bwd(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, scratch, scratch_bytes, stream=0):
    _check(lib().fcp_attn_bwd(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq), _ptr(dk),
                              _ptr(dv), _ptr(scratch), int(scratch_bytes), C.c_void_p(stream)))


def fcp_attn_bwd_heads(plan: Plan, q, k, v, o, d_o, lse, kv_head_begin, kv_head_count, dq, dk, dv, scratch, scratch_bytes,
                       stream=0):
    _check(lib().fcp_attn_bwd_heads(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), int(kv_head_begin),
                                    int(kv_head_count), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(scratch), int(scratch_bytes),
                                    C.c_void_p(stream)))


def fcp_attn_fwd_bwd_host(plan: Plan, q, k, v, d_o, o, lse, dq, dk, dv, workspace, workspace_bytes, stream=0):
    _check(lib().fcp_attn_fwd_bwd_host(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(d_o), _ptr(o), _ptr(lse), _ptr(dq),
                                       _ptr(dk), _ptr(dv), _ptr(workspace), int(workspace_bytes), C.c_void_p(stream)))


# ---------------------------------------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------------------------------------
ROPE_LAYOUTS = dict(half=0, interleaved=1)
ROPE_SCALINGS = dict(none=0, linear=1, ntk=2, yarn=3, wavelength=4)


class RopeTable:
    """Frequencies of fcp_rope_fwd / fcp_rope_bwd (fcp_rope_init)."""

    def __init__(self, head_dim, rotary_dim=None, layout="half", base=10000.0, scaling="none", factor=1.0, original_length=0.0,
                 low=0.0, high=0.0, magnitude=0.0):
        config = FcpRopeConfig(int(head_dim), int(head_dim if rotary_dim is None else rotary_dim), _named(ROPE_LAYOUTS, layout),
                               _named(ROPE_SCALINGS, scaling), float(base), float(factor), float(original_length), float(low),
                               float(high), float(magnitude))
        _torch_types()
        self.struct = FcpRopeTable()
        _check(lib().fcp_rope_init(C.byref(config), C.byref(self.struct)))
        self.ref, self.head_dim = C.byref(self.struct), self.struct.head_dim

    def frequencies(self) -> np.ndarray:
        """Radians per token of each pair, as the table holds them."""
        turns = np.asarray(self.struct.turn[:self.struct.rotary_dim // 2], dtype=np.uint64)
        return turns.astype(np.float64) * (2.0 * np.pi / 2.0 ** 64)


def _named(names: dict, value) -> int:
    """The number of a name; a number as it is."""
    if isinstance(value, str):
        if value not in names:
            raise ValueError(f"{value!r} is none of {', '.join(names)}")
        return names[value]
    return int(value)


# The checks below stand in front of kernels of a few microseconds: one look at type, shape, strides and device per tensor, no
# conversions.  A tensor of another type would be read as what it is not, and one of another place is no address on this GPU.
_BF16 = _F32 = _I32 = None


def _torch_types():
    """Called where a table, a cache or a batch is made: PyTorch need not be there for the planner's calls."""
    global _BF16, _F32, _I32
    if _BF16 is None:
        import torch
        _BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32


def _heads(x, head_dim, name):
    """Rows, heads, row stride, address and device of a bf16 tensor [rows][heads][head_dim] whose heads are contiguous."""
    rows, heads, d = x.shape
    s0, s1, s2 = x.stride()
    if d != head_dim or s2 != 1 or (s1 != d and heads > 1) or x.dtype is not _BF16:
        raise ValueError(f"{name}: a bf16 tensor [rows][heads][{head_dim}] with contiguous heads is wanted")
    if rows <= 1:
        s0 = heads * d
    elif s0 < heads * d:                           # an expanded tensor: its stride 0 means heads * head_dim to the library
        raise ValueError(f"{name}: rows that share memory (row stride {s0}); a row of its own for each is wanted, see Tensor.contiguous")
    return rows, heads, s0, x.data_ptr(), x.get_device()


_NO_HEADS = (None, 0, 0, None, None)


def _i32_ptr(x, n, name, device=None):
    """Address of a contiguous int32 device tensor of n entries (None: NULL), of that device if one is given."""
    if x is None:
        return None
    if x.dtype is not _I32 or x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor of {n} entries is wanted")
    if device is not None and x.get_device() != device:
        _elsewhere(device)
    return x.data_ptr()


def _elsewhere(device):
    raise ValueError("the tensors of a call are wanted on one GPU" + (f", here cuda:{device}" if device >= 0 else ""))


_ONE_DEVICE = None                                 # whether there is one GPU only; not known yet


def _not_current(device) -> bool:
    global _ONE_DEVICE
    import torch
    if _ONE_DEVICE is None:
        _ONE_DEVICE = torch.cuda.device_count() == 1
    return not _ONE_DEVICE and device != torch.cuda.current_device()


def _rope(call, table, q, k, q_out, k_out, positions, row_offset, length, stream):
    d = table.head_dim
    rows, hq, qs, qp, qd = _NO_HEADS if q is None else _heads(q, d, "q")
    k_rows, hkv, ks, kp, kd = _NO_HEADS if k is None else _heads(k, d, "k")
    q_out_rows, hq_out, qos, qop, qod = _NO_HEADS if q_out is None else _heads(q_out, d, "q_out")
    k_out_rows, hkv_out, kos, kop, kod = _NO_HEADS if k_out is None else _heads(k_out, d, "k_out")
    if hq_out != hq or hkv_out != hkv or q_out_rows != rows or k_out_rows != k_rows or (q is not None and k is not None and k_rows != rows):
        raise ValueError("q, k, q_out, k_out differ in rows or heads")
    T = rows or k_rows or 0
    B = 0 if row_offset is None else row_offset.numel() - 1
    device = None
    if T:
        device = kd if qd is None else qd
        if device < 0 or qod != qd or kod != kd or (qd is not None and kd is not None and kd != qd):
            _elsewhere(device)
    positions, row_offset, length = (_i32_ptr(positions, T, "positions", device), _i32_ptr(row_offset, B + 1, "row_offset", device),
                                     _i32_ptr(length, B, "length", device))
    if T and not _ONE_DEVICE and _not_current(device):
        raise ValueError(f"the tensors lie on cuda:{device}, which is not the current device")
    rc = call(table.ref, T, qp, qs, hq, kp, ks, hkv, qop, qos, kop, kos, positions, row_offset, length, B, stream)
    if rc:
        _check(rc)


def fcp_rope_fwd(table: RopeTable, q, k, q_out, k_out, positions=None, row_offset=None, length=None, stream=0):
    """q, k and their outputs: bf16 [T][heads][head_dim] (slices of wider rows are fine; outputs may be the inputs); either
    pair may be None.  Positions are given, or follow from the batch's row_offset (and the sequences' lengths; not after an eviction,
    which shortens them and leaves the kept keys' positions as they were)."""
    _rope(lib().fcp_rope_fwd, table, q, k, q_out, k_out, positions, row_offset, length, stream)


def fcp_rope_bwd(table: RopeTable, dq, dk, dq_in, dk_in, positions=None, row_offset=None, length=None, stream=0):
    """Gradients of the outputs dq, dk -> gradients of the inputs dq_in, dk_in; arguments as in fcp_rope_fwd."""
    _rope(lib().fcp_rope_bwd, table, dq, dk, dq_in, dk_in, positions, row_offset, length, stream)


# ---------------------------------------------------------------------------------------------------------
# Cache of keys and values in 8 bits
# ---------------------------------------------------------------------------------------------------------
CACHE_KINDS = dict(e4m3=0, int8=1)
FCP_CACHE_MIN_SCALE, FCP_CACHE_MAX_SCALE = 2.0 ** -100, 2.0 ** 122
FCP_CACHE_BAD_LENGTH, FCP_CACHE_BAD_ROWS, FCP_CACHE_BAD_PAGE, FCP_CACHE_BAD_SCALE = 1001, 1002, 1003, 1004


class Cache:
    """Owns an fcp_cache handle over the caller's pages: k, v [n_pages][hkv][page_tokens][head_dim] (float8_e4m3fn or int8),
    k_scale, v_scale fp32 [n_pages][hkv], status int32 [4] (zeroed), weight fp32 [n_pages][hkv][page_tokens] or None."""

    def __init__(self, k, v, k_scale, v_scale, status, weight=None, kind=None):
        _torch_types()
        n_pages, hkv, page_tokens, head_dim = k.shape
        if kind is None:
            kind = {"torch.float8_e4m3fn": "e4m3", "torch.int8": "int8"}.get(str(k.dtype))
            if kind is None:
                raise ValueError(f"pages of {k.dtype}: say which kind of code they hold")
        for x, shape, dtype in ((k, k.shape, None), (v, k.shape, None), (k_scale, (n_pages, hkv), _F32), (v_scale, (n_pages, hkv), _F32),
                                (weight, (n_pages, hkv, page_tokens), _F32), (status, (4,), _I32)):
            if x is not None and (tuple(x.shape) != tuple(shape) or not x.is_contiguous() or not (x.dtype is dtype if dtype else x.dtype.itemsize == 1)):
                raise ValueError(f"a contiguous tensor {tuple(shape)} of {dtype or '1-byte values'} is wanted, not {tuple(x.shape)} {x.dtype}")
        self.device = k.get_device()                 # -1: host memory, which the library's calls refuse
        if any(x is not None and x.get_device() != self.device for x in (v, k_scale, v_scale, status, weight)):
            raise ValueError("the tensors of a cache lie on different devices")
        self.hkv, self.head_dim, self.page_tokens, self.n_pages = hkv, head_dim, page_tokens, n_pages
        self.tensors = (k, v, k_scale, v_scale, status, weight)          # the pages live as long as the handle
        ptr = [None if x is None else x.data_ptr() for x in (k, v, k_scale, v_scale, weight, status)]
        config = FcpCacheConfig(*ptr, n_pages, page_tokens, hkv, head_dim, _named(CACHE_KINDS, kind))
        self.handle = C.c_void_p()
        _check(lib().fcp_cache_create(C.byref(config), C.byref(self.handle)))

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value and _lib is not None:
            _lib.fcp_cache_destroy(h)
            self.handle = None

    def device_status(self):
        st = np.zeros(4, dtype=np.int32)
        _check(lib().fcp_cache_device_status(self.handle, st.ctypes.data_as(C.POINTER(C.c_int32))))
        return st


class CacheBatch:
    """The sequences a call works on: page_table int32 [B][width], length int32 [B] (new tokens included), row_offset int32 [B+1]
    (device tensors, read when the call runs); rows and max_new bound them.  max_new defaults to rows, which is right for one sequence
    only: the kernels of fcp_cache_attn are chosen by it, so a step of single tokens passes max_new=1."""

    def __init__(self, page_table, length, row_offset=None, rows=0, max_new=None):
        _torch_types()
        B, width = page_table.shape
        self.tensors = (page_table, length, row_offset)
        self.device = page_table.get_device()
        if any(x is not None and x.get_device() != self.device for x in (length, row_offset)):
            raise ValueError("the tensors of a batch lie on different devices")
        self.B, self.rows = B, int(rows)
        self.struct = FcpCacheBatch(B, self.rows, int(rows if max_new is None else max_new), width,
                                    _i32_ptr(page_table, B * width, "page_table"), _i32_ptr(length, B, "length"),
                                    _i32_ptr(row_offset, B + 1, "row_offset"))
        self.ref = C.byref(self.struct)


def _on_cache(cache: Cache, batch: CacheBatch, *devices):
    """Everything where the pages are.  (Pages in host memory are left to the library, which refuses them.)"""
    device = cache.device
    if device >= 0:
        if batch.device != device:
            raise ValueError(f"the cache lies on cuda:{device}, the batch does not")
        for d in devices:
            if d != device:
                _elsewhere(device)


def fcp_cache_append(cache: Cache, batch: CacheBatch, k, v, stream=0):
    k_rows, k_heads, ks, kp, kd = _heads(k, cache.head_dim, "k")
    v_rows, v_heads, vs, vp, vd = _heads(v, cache.head_dim, "v")
    if k_rows != batch.rows or v_rows != batch.rows or k_heads != cache.hkv or v_heads != cache.hkv:
        raise ValueError(f"k, v: {batch.rows} rows of {cache.hkv} heads are wanted")
    _on_cache(cache, batch, kd, vd)
    rc = lib().fcp_cache_append(cache.handle, batch.ref, kp, ks, vp, vs, stream)
    if rc:
        _check(rc)


def fcp_cache_attn_workspace_bytes(cache: Cache, batch: CacheBatch, hq) -> int:
    v = C.c_int64(0)
    _check(lib().fcp_cache_attn_workspace_bytes(cache.handle, batch.ref, int(hq), C.byref(v)))
    return v.value


def fcp_cache_attn(cache: Cache, batch: CacheBatch, q, o, lse, workspace, workspace_bytes, scale=0.0, accumulate=False, stream=0):
    rows, hq, qs, qp, qd = _heads(q, cache.head_dim, "q")
    o_rows, o_heads, _, op, od = _heads(o, cache.head_dim, "o")
    if rows != batch.rows or o_rows != rows or o_heads != hq or not o.is_contiguous():
        raise ValueError(f"q, o: {batch.rows} rows of the same heads are wanted, o contiguous")
    if lse.numel() != rows * hq or lse.dtype is not _F32 or not lse.is_contiguous():
        raise ValueError("lse: a contiguous fp32 tensor [rows][hq] is wanted")
    wd = cache.device if workspace is None else workspace.get_device()
    if workspace is not None and (workspace.nbytes < workspace_bytes or not workspace.is_contiguous()):
        raise ValueError(f"workspace: contiguous, of at least the {workspace_bytes} bytes that the call names")
    _on_cache(cache, batch, qd, od, lse.get_device(), wd)
    rc = lib().fcp_cache_attn(cache.handle, batch.ref, qp, qs, hq, scale, op, lse.data_ptr(), 1 if accumulate else 0,
                              None if workspace is None else workspace.data_ptr(), workspace_bytes, stream)
    if rc:
        _check(rc)


def fcp_cache_evict(cache: Cache, batch: CacheBatch, n_sink, n_heavy, n_recent, dst_table, new_length, kept, stream=0):
    B, width = dst_table.shape
    if B != batch.B:
        raise ValueError("dst_table and the batch differ in their number of sequences")
    keep = int(n_sink) + int(n_heavy) + int(n_recent)
    _on_cache(cache, batch, dst_table.get_device(), new_length.get_device(), kept.get_device())
    _check(lib().fcp_cache_evict(cache.handle, batch.ref, int(n_sink), int(n_heavy), int(n_recent),
                                 _i32_ptr(dst_table, B * width, "dst_table"), width, _i32_ptr(new_length, B, "new_length"),
                                 _i32_ptr(kept, B * cache.hkv * keep, "kept"), stream))


FCP_NOALLOC_MAX_BYTES = 32 << 20


def fcp_noalloc_bytes_needed(plan: Plan) -> int:
    v = C.c_int64(0)
    _check(lib().fcp_noalloc_bytes_needed(plan.handle, C.byref(v)))
    return v.value


def fcp_attn_bwd_noalloc(plan: Plan, q, k, v, o, d_o, lse, dq, dk, dv, stream=0):
    """Backward pass that allocates nothing: the plan need not be uploaded and no scratch is passed;
    the library's built-in arena (FCP_NOALLOC_MAX_BYTES per GPU) holds tables and scratch."""
    _check(lib().fcp_attn_bwd_noalloc(plan.handle, _ptr(q), _ptr(k), _ptr(v), _ptr(o), _ptr(d_o), _ptr(lse), _ptr(dq),
                                      _ptr(dk), _ptr(dv), C.c_void_p(stream)))


def fcp_noalloc_device_status():
    st = np.zeros(4, dtype=np.int32)
    _check(lib().fcp_noalloc_device_status(st.ctypes.data_as(C.POINTER(C.c_int32))))
    return st


def fcp_selftest_bounded_wait(limit_us=1000, stream=0):
    """Makes one bounded device-side wait run out on purpose (a barrier nobody arrives at, limit in
    microseconds) and returns the four status words it produced."""
    st = np.zeros(4, dtype=np.int32)
    _check(lib().fcp_selftest_bounded_wait(int(limit_us), st.ctypes.data_as(C.POINTER(C.c_int32)), C.c_void_p(stream)))
    return st
