"""Thin ctypes binding of libhifa4 (the C ABI declared in include/hifa4.h).

Argument marshalling only: every step of the path runs in the CUDA kernels of the library.
torch supplies device memory and the current stream.  There is no CPU fallback: if the shared
library is missing or cannot be loaded, every call raises."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from functools import lru_cache

import torch

from . import build as _build

F16, BF16, F32 = 0, 1, 2
Q, K, V = 0, 1, 2
CODES, META, MMA, AUX = 0, 1, 2, 3
MODE_BYPASS, MODE_STRONG, MODE_MILD, MODE_AUTO, MODE_CUSTOM = 0, 1, 2, 3, 4
AGG_RMS, AGG_MEAN, AGG_P99 = 0, 0x100, 0x200            # OR-ed into the calibration mode
MAX_DEBUG_BLOCKS = 16

_DT = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}
_TORCH_DT = {F16: torch.float16, BF16: torch.bfloat16, F32: torch.float32}


class Hifa4Error(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class _Shape(C.Structure):
    _fields_ = [("B", C.c_int), ("Hq", C.c_int), ("Hkv", C.c_int), ("N", C.c_int), ("d", C.c_int),
                ("q_to_kv", C.POINTER(C.c_int)), ("in_dtype", C.c_int)]


class _QKV(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q_codes", "q_meta", "q_mma", "k_codes", "k_meta", "k_mma",
                                          "v_codes", "v_meta", "v_mma", "q_mu", "k_sum")]


class _AttnParams(C.Structure):
    _fields_ = [("causal", C.c_int), ("Br", C.c_int), ("Bc", C.c_int), ("normalizer", C.c_int),
                ("qmean", C.c_int), ("p_dtype", C.c_int), ("out_dtype", C.c_int),
                ("softmax_scale", C.c_float)]


class _Debug(C.Structure):
    _fields_ = [("n_blocks", C.c_int), ("blocks", C.POINTER(C.c_int)), ("p_codes", C.c_void_p),
                ("p_step", C.c_void_p), ("l_out", C.c_void_p), ("m_out", C.c_void_p)]


class _CalibStats(C.Structure):
    _fields_ = [("rho_K", C.c_float), ("T_KQ", C.c_float), ("branch", C.c_int), ("alpha", C.c_float)]


class _MassStats(C.Structure):
    _fields_ = [("hist", C.c_void_p), ("n_bins", C.c_int), ("lo", C.c_double), ("hi", C.c_double)]


class _Cache(C.Structure):
    _fields_ = [("Hkv", C.c_int), ("d", C.c_int), ("in_dtype", C.c_int), ("n_pages", C.c_int), ("pages", C.c_void_p),
                ("n_tails", C.c_int), ("v_tail", C.c_void_p)]


class _Seqs(C.Structure):
    _fields_ = [("B", C.c_int), ("max_pages", C.c_int), ("block_table", C.c_void_p), ("kv_lens", C.c_void_p),
                ("tail_slots", C.c_void_p)]


class _Strides(C.Structure):
    _fields_ = [("b", C.c_longlong), ("h", C.c_longlong), ("t", C.c_longlong)]


class _CacheQuery(C.Structure):
    _fields_ = [("Hq", C.c_int), ("q_to_kv", C.POINTER(C.c_int)), ("N", C.c_int), ("causal", C.c_int), ("out_dtype", C.c_int),
                ("softmax_scale", C.c_float)]


_lib = None


def lib_path() -> str:
    return _build.LIB


def lib():
    """Load libhifa4.so (built in-tree by paper_2607_04302_b200.build).  Raises if it is absent."""
    global _lib
    if _lib is None:
        path = lib_path()
        if not os.path.exists(path):
            raise FileNotFoundError(
                f"{path} not found: build it with `python -m paper_2607_04302_b200.build` "
                "(the HiFA4 path has no CPU fallback)")
        L = C.CDLL(path)
        L.hifa4_status_string.restype = C.c_char_p
        L.hifa4_status_string.argtypes = [C.c_int]
        L.hifa4_get_counters.restype = None
        L.hifa4_quant_bytes.restype = C.c_size_t
        L.hifa4_quant_bytes.argtypes = [C.POINTER(_Shape), C.c_int, C.c_int]
        L.hifa4_attention_workspace_bytes.restype = C.c_size_t
        L.hifa4_attention_workspace_bytes.argtypes = [C.POINTER(_Shape), C.POINTER(_AttnParams)]
        L.hifa4_attention_raw_workspace_bytes.restype = C.c_size_t
        L.hifa4_attention_raw_workspace_bytes.argtypes = [C.POINTER(_Shape), C.POINTER(_AttnParams)]
        L.hifa4_smooth_calibrate.restype = C.c_int
        L.hifa4_smooth_calibrate.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int,
                                             C.c_int, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_float,
                                             C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(_CalibStats),
                                             C.c_void_p]
        L.hifa4_smooth_calibrate_auto.restype = C.c_int
        L.hifa4_smooth_calibrate_auto.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int,
                                                  C.c_int, C.POINTER(C.c_int), C.c_int, C.c_void_p, C.c_void_p,
                                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.hifa4_smooth_calibrate_static.restype = C.c_int
        L.hifa4_smooth_calibrate_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int,
                                                    C.c_int, C.POINTER(C.c_int), C.c_int, C.c_int, C.c_float,
                                                    C.c_void_p, C.c_void_p, C.POINTER(_CalibStats), C.c_void_p]
        L.hifa4_quantize_qkv.restype = C.c_int
        L.hifa4_quantize_qkv.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.POINTER(_QKV), C.c_void_p, C.c_void_p]
        L.hifa4_attention_fwd.restype = C.c_int
        L.hifa4_attention_fwd.argtypes = [C.POINTER(_Shape), C.POINTER(_QKV), C.POINTER(_AttnParams),
                                          C.c_void_p, C.c_void_p, C.POINTER(_Debug), C.c_void_p, C.c_void_p]
        L.hifa4_attention_fwd_qraw.restype = C.c_int
        L.hifa4_attention_fwd_qraw.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.POINTER(_QKV),
                                               C.POINTER(_AttnParams), C.c_void_p, C.c_void_p, C.c_void_p,
                                               C.c_void_p]
        L.hifa4_f8qk_workspace_bytes.restype = C.c_size_t
        L.hifa4_f8qk_workspace_bytes.argtypes = [C.POINTER(_Shape)]
        L.hifa4_attention_fwd_f8qk.restype = C.c_int
        L.hifa4_attention_fwd_f8qk.argtypes = [C.POINTER(_Shape), C.POINTER(_QKV), C.POINTER(_AttnParams), C.c_void_p,
                                               C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.hifa4_selftest_wait_timeout.restype = C.c_int
        L.hifa4_selftest_wait_timeout.argtypes = [C.POINTER(_Shape), C.POINTER(_QKV), C.POINTER(_AttnParams),
                                                  C.c_void_p, C.c_void_p, C.c_void_p]
        L.hifa4_attention_fwd_stats.restype = C.c_int
        L.hifa4_attention_fwd_stats.argtypes = [C.POINTER(_Shape), C.POINTER(_QKV), C.POINTER(_AttnParams),
                                                C.c_void_p, C.c_void_p, C.POINTER(_MassStats), C.c_void_p,
                                                C.c_void_p]
        L.hifa4_attention_fwd_raw.restype = C.c_int
        L.hifa4_attention_fwd_raw.argtypes = [C.POINTER(_Shape), C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_void_p, C.POINTER(_AttnParams), C.c_void_p,
                                              C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        P, I, V = C.POINTER, C.c_int, C.c_void_p
        L.hifa4_cache_page_bytes.restype = C.c_size_t
        L.hifa4_cache_page_bytes.argtypes = [I]
        L.hifa4_cache_append.restype = I
        L.hifa4_cache_append.argtypes = [P(_Cache), P(_Seqs), I, V, V, P(_Strides), V, P(_Strides), V, V, V]
        L.hifa4_cache_read.restype = I
        L.hifa4_cache_read.argtypes = [P(_Cache), P(_Seqs), I, V, I, V, V, V, V]
        L.hifa4_cache_decode_workspace_bytes.restype = C.c_size_t
        L.hifa4_cache_decode_workspace_bytes.argtypes = [P(_Cache), I, I, P(_CacheQuery), I]
        L.hifa4_cache_decode.restype = I
        L.hifa4_cache_decode.argtypes = [P(_Cache), P(_Seqs), P(_CacheQuery), V, P(_Strides), V, V, V, V, V, V, C.c_size_t, V, V]
        L.hifa4_cache_attention_workspace_bytes.restype = C.c_size_t
        L.hifa4_cache_attention_workspace_bytes.argtypes = [P(_Cache), I, I, P(_CacheQuery)]
        L.hifa4_cache_attention.restype = I
        L.hifa4_cache_attention.argtypes = [P(_Cache), P(_Seqs), P(_CacheQuery), V, P(_Strides), V, V, V, C.c_size_t, V, V]
        L.hifa4_selftest_cache_wait_timeout.restype = I
        L.hifa4_selftest_cache_wait_timeout.argtypes = [P(_Cache), P(_Seqs), P(_CacheQuery), V, V, V, V, C.c_size_t, V, V]
        L.hifa4_cache_evict.restype = I
        L.hifa4_cache_evict.argtypes = [P(_Seqs), V, I, I, I, V, V, V, V, V, V, V]
        _lib = L
    return _lib


STATIC_CALIB_MAX_FLOATS = 1 << 20

EXPORTS = ("hifa4_status_string", "hifa4_get_counters", "hifa4_smooth_calibrate",
           "hifa4_smooth_calibrate_static", "hifa4_smooth_calibrate_auto", "hifa4_quant_bytes",
           "hifa4_quantize_qkv", "hifa4_attention_workspace_bytes", "hifa4_attention_fwd",
           "hifa4_attention_fwd_stats", "hifa4_attention_raw_workspace_bytes", "hifa4_attention_fwd_raw",
           "hifa4_attention_fwd_qraw", "hifa4_f8qk_workspace_bytes", "hifa4_attention_fwd_f8qk",
           "hifa4_selftest_wait_timeout", "hifa4_cache_page_bytes", "hifa4_cache_append", "hifa4_cache_read",
           "hifa4_cache_decode_workspace_bytes", "hifa4_cache_decode", "hifa4_cache_attention_workspace_bytes",
           "hifa4_cache_attention", "hifa4_cache_evict", "hifa4_selftest_cache_wait_timeout")


def status_string(status: int) -> str:
    return lib().hifa4_status_string(int(status)).decode()


def get_counters():
    arr = (C.c_ulonglong * 4)()
    lib().hifa4_get_counters(arr)
    return dict(calibrate=arr[0], quantize=arr[1], attention=arr[2], launches=arr[3])


def _check(rc: int, where: str):
    if rc != 0:
        raise Hifa4Error(rc, where)


# Host time per call matters for short prompts (two launches of 4 and 8 us): pointers travel as plain integers (argtypes
# turn them into void*), the stream is read as a handle (0.2 us; building a torch.cuda.Stream object takes 3.3 us), and
# outputs come from empty_like (1.4 us against 2.4 us for torch.empty with a shape) where a tensor of their shape is at hand
# (the buffers of a QuantizedQKV may be flat views of an arena, of any element type).
def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _empty_out(like, out_dtype):
    """Contiguous uninitialised tensor of `like`'s shape and device."""
    return torch.empty_like(like, dtype=_TORCH_DT[out_dtype], memory_format=torch.contiguous_format)


def _map_arr(q_to_kv):
    if q_to_kv is None:
        return None, None
    arr = (C.c_int * len(q_to_kv))(*[int(x) for x in q_to_kv])
    return arr, C.cast(arr, C.POINTER(C.c_int))


def _shape(B, Hq, Hkv, N, d, in_dtype, q_to_kv=None):
    keep, p = _map_arr(q_to_kv)
    s = _Shape(B, Hq, Hkv, N, d, p, in_dtype)
    s._keep = keep
    return s


def _params(causal, Bc, out_dtype, Br=128, normalizer=0, qmean=0, p_dtype=F16, softmax_scale=0.0):
    return _AttnParams(int(causal), Br, Bc, normalizer, qmean, p_dtype, out_dtype, float(softmax_scale))


@dataclass
class QuantizedQKV:
    """Device buffers of one hifa4_qkv (see include/hifa4.h for the layouts)."""
    B: int
    Hq: int
    Hkv: int
    N: int
    d: int
    in_dtype: int
    q_to_kv: object
    q_codes: torch.Tensor
    q_meta: torch.Tensor
    q_mma: torch.Tensor
    k_codes: torch.Tensor
    k_meta: torch.Tensor
    k_mma: torch.Tensor
    v_codes: torch.Tensor
    v_meta: torch.Tensor
    v_mma: torch.Tensor
    q_mu: torch.Tensor | None = None        # Q-Mean auxiliary: per-token mean of the smoothed query
    k_sum: torch.Tensor | None = None       # Q-Mean auxiliary: channel sum of the smoothed key

    def struct(self) -> _QKV:
        return _QKV(self.q_codes.data_ptr(), self.q_meta.data_ptr(), self.q_mma.data_ptr(),
                    self.k_codes.data_ptr(), self.k_meta.data_ptr(), self.k_mma.data_ptr(),
                    self.v_codes.data_ptr(), self.v_meta.data_ptr(), self.v_mma.data_ptr(),
                    _ptr(self.q_mu), _ptr(self.k_sum))


def quant_bytes(B, Hq, Hkv, N, d, in_dtype, which, part) -> int:
    s = _shape(B, Hq, Hkv, N, d, in_dtype)
    return int(lib().hifa4_quant_bytes(C.byref(s), which, part))


def alloc_qkv(B, Hq, Hkv, N, d, in_dtype, device, q_to_kv=None, qmean=False) -> QuantizedQKV:
    """Allocate the buffers with the sizes the library reports (qmean: also the two Q-Mean vectors)."""
    bufs = {}
    size = lib().hifa4_quant_bytes
    sh = C.byref(_shape(B, Hq, Hkv, N, d, in_dtype))
    for w, name, H in ((Q, "q", Hq), (K, "k", Hkv), (V, "v", Hkv)):
        nb = [size(sh, w, p) for p in (CODES, META, MMA)]
        if 0 in nb:
            raise Hifa4Error(2, "hifa4_quant_bytes")
        tok_axis = (w == V)
        lead = (B, H, d) if tok_axis else (B, H, N)
        ln = N if tok_axis else d
        bufs[name + "_codes"] = torch.empty(lead + (ln // 2,), dtype=torch.uint8, device=device)
        bufs[name + "_meta"] = torch.empty(lead + (ln // 64,), dtype=torch.int32, device=device)
        bufs[name + "_mma"] = torch.empty(lead + (ln,), dtype=torch.bfloat16, device=device)
        assert bufs[name + "_codes"].numel() == nb[0] and bufs[name + "_meta"].numel() * 4 == nb[1]
        assert bufs[name + "_mma"].numel() * 2 == nb[2]
    if qmean:
        assert quant_bytes(B, Hq, Hkv, N, d, in_dtype, Q, AUX) == B * Hq * N * 4
        bufs["q_mu"] = torch.empty((B, Hq, N), dtype=torch.float32, device=device)
        bufs["k_sum"] = torch.empty((B, Hkv, N), dtype=torch.float32, device=device)
    return QuantizedQKV(B, Hq, Hkv, N, d, in_dtype, q_to_kv, **bufs)


def smooth_calibrate(q_cal, k_cal, mode, alpha=0.0, q_to_kv=None, aggregator=AGG_RMS):
    """q_cal [S,Hq,Ncal,d], k_cal [S,Hkv,Ncal,d] device tensors -> (s, inv_s) [Hkv,d] float32.
    aggregator: AGG_RMS (the paper's choice), AGG_MEAN or AGG_P99 over the calibration samples."""
    assert q_cal.is_cuda and k_cal.is_cuda and q_cal.is_contiguous() and k_cal.is_contiguous()
    S, Hq, Ncal, d = q_cal.shape
    Hkv = k_cal.shape[1]
    dev = q_cal.device
    s = torch.empty((Hkv, d), dtype=torch.float32, device=dev)
    inv_s = torch.empty_like(s)
    ws = torch.empty((2, S, Hkv, d), dtype=torch.float32, device=dev)
    keep, mp = _map_arr(q_to_kv)
    stats = _CalibStats()
    rc = lib().hifa4_smooth_calibrate(_ptr(q_cal), _ptr(k_cal), S, Hq, Hkv, Ncal, d, mp, _DT[q_cal.dtype],
                                      int(mode) | int(aggregator), float(alpha), _ptr(s), _ptr(inv_s), _ptr(ws),
                                      C.byref(stats), _stream())
    _check(rc, "hifa4_smooth_calibrate")
    return s, inv_s


GATE_WS_BYTES = 32768 * 4 + 64


def smooth_calibrate_auto(q_cal, k_cal, q_to_kv=None):
    """Calibration with the applicability gate deciding the branch on the device.
    Returns (s, inv_s, stats) with stats a DEVICE float32 tensor [rho_K, T_K/Q, branch, alpha]."""
    assert q_cal.is_cuda and k_cal.is_cuda and q_cal.is_contiguous() and k_cal.is_contiguous()
    S, Hq, Ncal, d = q_cal.shape
    Hkv = k_cal.shape[1]
    dev = q_cal.device
    s = torch.empty((Hkv, d), dtype=torch.float32, device=dev)
    inv_s = torch.empty_like(s)
    ws = torch.empty((2, S, Hkv, d), dtype=torch.float32, device=dev)
    gate_ws = torch.empty(GATE_WS_BYTES // 8, dtype=torch.int64, device=dev)
    stats = torch.empty(4, dtype=torch.float32, device=dev)
    keep, mp = _map_arr(q_to_kv)
    rc = lib().hifa4_smooth_calibrate_auto(_ptr(q_cal), _ptr(k_cal), S, Hq, Hkv, Ncal, d, mp, _DT[q_cal.dtype],
                                           _ptr(s), _ptr(inv_s), _ptr(ws), _ptr(gate_ws), _ptr(stats), _stream())
    _check(rc, "hifa4_smooth_calibrate_auto")
    return s, inv_s, stats


def smooth_calibrate_static(q_cal, k_cal, mode, alpha=0.0, q_to_kv=None, s=None, inv_s=None):
    """smooth_calibrate through the entry point that allocates nothing on the device: the scratch
    is the library's fixed array (2*S*Hkv*d <= STATIC_CALIB_MAX_FLOATS, else Hifa4Error with status
    3).  The caller may pass preallocated outputs s, inv_s [Hkv,d] float32; they are created here
    only for convenience when omitted (the C entry point itself never allocates)."""
    assert q_cal.is_cuda and k_cal.is_cuda and q_cal.is_contiguous() and k_cal.is_contiguous()
    S, Hq, Ncal, d = q_cal.shape
    Hkv = k_cal.shape[1]
    if s is None:
        s = torch.empty((Hkv, d), dtype=torch.float32, device=q_cal.device)
    if inv_s is None:
        inv_s = torch.empty_like(s)
    keep, mp = _map_arr(q_to_kv)
    stats = _CalibStats()
    rc = lib().hifa4_smooth_calibrate_static(_ptr(q_cal), _ptr(k_cal), S, Hq, Hkv, Ncal, d, mp,
                                             _DT[q_cal.dtype], int(mode), float(alpha), _ptr(s), _ptr(inv_s),
                                             C.byref(stats), _stream())
    _check(rc, "hifa4_smooth_calibrate_static")
    return s, inv_s


def quantize_qkv(q, k, v, s=None, inv_s=None, q_to_kv=None, out: QuantizedQKV | None = None,
                 d_status=None, qmean=False, Hq=None) -> QuantizedQKV:
    """Smooth-QK + HIF4 quantization of device tensors q [B,Hq,N,d], k, v [B,Hkv,N,d].
    qmean: also apply the Q-Mean auxiliary (the Q buffers then hold the mean-free Q_z).
    q = None: K and V only (for attention_fwd_qraw); Hq then names the number of query heads."""
    assert k.is_cuda and k.is_contiguous() and v.is_contiguous() and (q is None or q.is_contiguous())
    if q is None:
        assert Hq is not None and not qmean
        B, _, N, d = k.shape
    else:
        B, Hq, N, d = q.shape
    Hkv = k.shape[1]
    dt = _DT[k.dtype]
    if out is None:
        out = alloc_qkv(B, Hq, Hkv, N, d, dt, k.device, q_to_kv, qmean=qmean)
    sh = _shape(B, Hq, Hkv, N, d, dt, q_to_kv)
    st = out.struct()
    rc = lib().hifa4_quantize_qkv(C.byref(sh), _ptr(q), _ptr(k), _ptr(v), _ptr(s), _ptr(inv_s),
                                  C.byref(st), _ptr(d_status), _stream())
    _check(rc, "hifa4_quantize_qkv")
    return out


def attention_fwd(qkv: QuantizedQKV, causal: bool, Bc: int = 64, out_dtype=F32, out=None,
                  debug_blocks=None, d_status=None, softmax_scale=0.0, Br=128, qmean=False, normalizer=0,
                  p_dtype=F16):
    """Fused attention forward on quantized operands.  Returns out [B,Hq,N,d], or
    (out, dict(p_codes, p_step, l, m)) when debug_blocks (a list of (b, h, query block)) is given."""
    dev = qkv.q_mma.device
    sh = _shape(qkv.B, qkv.Hq, qkv.Hkv, qkv.N, qkv.d, qkv.in_dtype, qkv.q_to_kv)
    prm = _params(causal, Bc, out_dtype, Br=Br, softmax_scale=softmax_scale, qmean=int(qmean),
                  normalizer=int(normalizer), p_dtype=p_dtype)
    if out is None:
        out = qkv.q_mma.new_empty((qkv.B, qkv.Hq, qkv.N, qkv.d), dtype=_TORCH_DT[out_dtype])
    st = qkv.struct()
    dbg_p, dump = None, None
    if debug_blocks:
        nb = len(debug_blocks)
        flat = (C.c_int * (3 * nb))(*[int(x) for t in debug_blocks for x in t])
        dump = dict(p_codes=torch.zeros((nb, 128, qkv.N), dtype=torch.uint8, device=dev),
                    p_step=torch.zeros((nb, 128, qkv.N // 4), dtype=torch.float32, device=dev),
                    l=torch.zeros((nb, 128), dtype=torch.float32, device=dev),
                    m=torch.zeros((nb, 128), dtype=torch.float32, device=dev))
        dbg = _Debug(nb, C.cast(flat, C.POINTER(C.c_int)), dump["p_codes"].data_ptr(),
                     dump["p_step"].data_ptr(), dump["l"].data_ptr(), dump["m"].data_ptr())
        dbg_p = C.byref(dbg)
    ws_bytes = int(lib().hifa4_attention_workspace_bytes(C.byref(sh), C.byref(prm)))
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=dev) if ws_bytes else None
    rc = lib().hifa4_attention_fwd(C.byref(sh), C.byref(st), C.byref(prm), _ptr(out), _ptr(ws), dbg_p,
                                   _ptr(d_status), _stream())
    _check(rc, "hifa4_attention_fwd")
    return (out, dump) if debug_blocks else out


def attention_fwd_qraw(q, s, kv: QuantizedQKV, causal: bool, out_dtype=F32, out=None, d_status=None,
                       softmax_scale=0.0, p_dtype=F16):
    """attention_fwd whose kernel smooths and quantizes the raw q [B,Hq,N,d] itself (s: [Hkv,d] or None); kv holds
    the K and V images from quantize_qkv(None, k, v, ...).  Bc = 64, d = 64 or 128, no Q-Mean."""
    assert q.is_cuda and q.is_contiguous() and _DT[q.dtype] == kv.in_dtype
    sh = _shape(kv.B, kv.Hq, kv.Hkv, kv.N, kv.d, kv.in_dtype, kv.q_to_kv)
    assert tuple(q.shape) == (kv.B, kv.Hq, kv.N, kv.d)
    prm = _params(causal, 64, out_dtype, softmax_scale=softmax_scale, p_dtype=p_dtype)
    if out is None:
        out = _empty_out(q, out_dtype)
    st = kv.struct()
    rc = lib().hifa4_attention_fwd_qraw(C.byref(sh), _ptr(q), _ptr(s), C.byref(st), C.byref(prm), _ptr(out), None,
                                        _ptr(d_status), _stream())
    _check(rc, "hifa4_attention_fwd_qraw")
    return out


def attention_fwd_f8qk(qkv: QuantizedQKV, causal: bool, out_dtype=F32, out=None, workspace=None, d_status=None,
                       softmax_scale=0.0):
    """attention_fwd with Q K^T issued as kind::f8f6f4 on E4M3 images (experiment; d = 128, Bc = 64)."""
    dev = qkv.k_mma.device
    sh = _shape(qkv.B, qkv.Hq, qkv.Hkv, qkv.N, qkv.d, qkv.in_dtype, qkv.q_to_kv)
    prm = _params(causal, 64, out_dtype, softmax_scale=softmax_scale)
    need = int(lib().hifa4_f8qk_workspace_bytes(C.byref(sh)))
    if need == 0:
        raise Hifa4Error(2, "hifa4_f8qk_workspace_bytes")
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if out is None:
        out = torch.empty((qkv.B, qkv.Hq, qkv.N, qkv.d), dtype=_TORCH_DT[out_dtype], device=dev)
    st = qkv.struct()
    rc = lib().hifa4_attention_fwd_f8qk(C.byref(sh), C.byref(st), C.byref(prm), _ptr(out), _ptr(workspace),
                                        workspace.numel(), _ptr(d_status), _stream())
    _check(rc, "hifa4_attention_fwd_f8qk")
    return out


def selftest_wait_timeout(qkv: QuantizedQKV, causal: bool, d_status, out=None):
    """Launches the self-test instantiation whose wait for P V runs out, of the kernel that attention_fwd would take (see
    include/hifa4.h).  d_status: device
    int32 tensor (zero on entry); afterwards it holds HIFA4_ERR_TIMEOUT + 16 * 7.  Returns the (unwritten) out."""
    sh = _shape(qkv.B, qkv.Hq, qkv.Hkv, qkv.N, qkv.d, qkv.in_dtype, qkv.q_to_kv)
    prm = _params(causal, 64, F32)
    if out is None:
        out = torch.empty((qkv.B, qkv.Hq, qkv.N, qkv.d), dtype=torch.float32, device=qkv.q_mma.device)
    st = qkv.struct()
    rc = lib().hifa4_selftest_wait_timeout(C.byref(sh), C.byref(st), C.byref(prm), _ptr(out), _ptr(d_status), _stream())
    _check(rc, "hifa4_selftest_wait_timeout")
    return out


def attention_fwd_stats(qkv: QuantizedQKV, causal: bool, n_bins: int, lo: float, hi: float, Bc: int = 64,
                        out_dtype=F32, hist=None, d_status=None, softmax_scale=0.0, qmean=False, normalizer=0):
    """Attention forward that also adds to the histogram of the per-(row, key tile) mass error of P-hat.
    Returns (out, hist) with hist a device int64 tensor of n_bins + 2 counters (last two: below lo, at or above hi)."""
    dev = qkv.q_mma.device
    sh = _shape(qkv.B, qkv.Hq, qkv.Hkv, qkv.N, qkv.d, qkv.in_dtype, qkv.q_to_kv)
    prm = _params(causal, Bc, out_dtype, softmax_scale=softmax_scale, qmean=int(qmean), normalizer=int(normalizer))
    out = torch.empty((qkv.B, qkv.Hq, qkv.N, qkv.d), dtype=_TORCH_DT[out_dtype], device=dev)
    if hist is None:
        hist = torch.zeros(n_bins + 2, dtype=torch.int64, device=dev)
    st = qkv.struct()
    stats = _MassStats(hist.data_ptr(), int(n_bins), float(lo), float(hi))
    rc = lib().hifa4_attention_fwd_stats(C.byref(sh), C.byref(st), C.byref(prm), _ptr(out), None,
                                         C.byref(stats), _ptr(d_status), _stream())
    _check(rc, "hifa4_attention_fwd_stats")
    return out, hist


def attention_raw_workspace_bytes(B, Hq, Hkv, N, d, in_dtype, causal, Bc, out_dtype=F32, qmean=False) -> int:
    sh = _shape(B, Hq, Hkv, N, d, in_dtype)
    prm = _params(causal, Bc, out_dtype, qmean=int(qmean))
    return int(lib().hifa4_attention_raw_workspace_bytes(C.byref(sh), C.byref(prm)))


def attention_fwd_raw(q, k, v, s, inv_s, causal: bool, Bc: int = 64, out_dtype=F32, q_to_kv=None,
                      out=None, workspace=None, d_status=None, softmax_scale=0.0, qmean=False):
    """Algorithm 1 end to end on raw device tensors (quantize into the workspace, then attend)."""
    B, Hq, N, d = q.shape
    Hkv = k.shape[1]
    dt = _DT[q.dtype]
    sh = _shape(B, Hq, Hkv, N, d, dt, q_to_kv)
    prm = _params(causal, Bc, out_dtype, softmax_scale=softmax_scale, qmean=int(qmean))
    need = int(lib().hifa4_attention_raw_workspace_bytes(C.byref(sh), C.byref(prm)))
    if need == 0:
        raise Hifa4Error(2, "hifa4_attention_raw_workspace_bytes")
    if workspace is None:
        workspace = q.new_empty(need, dtype=torch.uint8)
    if out is None:
        out = _empty_out(q, out_dtype)
    rc = lib().hifa4_attention_fwd_raw(C.byref(sh), _ptr(q), _ptr(k), _ptr(v), _ptr(s), _ptr(inv_s),
                                       C.byref(prm), _ptr(out), _ptr(workspace),
                                       workspace.numel(), _ptr(d_status), _stream())
    _check(rc, "hifa4_attention_fwd_raw")
    return out


# ---------------------------------------------------------------- paged HIF4 cache
PAGE_TOKENS = 64


@dataclass(frozen=True)
class PagedCache:
    """Pages of a HIF4 key-value cache and the raw values of the incomplete ones (layouts: include/hifa4.h).
    v_tail = None: a cache that is only read."""
    pages: torch.Tensor                     # uint8 [n_pages, Hkv, 74 d]
    v_tail: torch.Tensor | None = None      # [n_tails, Hkv, 64, d] of the activation dtype

    def __post_init__(self):
        pages, tail = self.pages, self.v_tail
        assert pages.is_cuda and pages.dtype == torch.uint8 and pages.dim() == 3 and pages.is_contiguous()
        n_pages, Hkv, nbytes = pages.shape
        assert nbytes % 74 == 0
        n_tails = 0
        if tail is not None:
            assert tail.get_device() == pages.get_device() and tail.is_contiguous() and tuple(tail.shape[1:]) == (Hkv, PAGE_TOKENS, nbytes // 74)
            n_tails = tail.shape[0]
        # the C descriptors, formed once: a call's host time counts
        make = lambda dt: _Cache(Hkv, nbytes // 74, dt, n_pages, pages.data_ptr(), n_tails, _ptr(tail))
        object.__setattr__(self, "_st", {dt: make(dt) for dt in (F16, BF16)})

    def struct(self, in_dtype, dev=None) -> _Cache:
        st, pages, tail = self._st[in_dtype], self.pages, self.v_tail
        assert st.pages == pages.data_ptr() and (tail is None or st.v_tail == tail.data_ptr())
        assert pages.get_device() == (_get_device() if dev is None else dev)
        return st


def cache_page_bytes(d) -> int:
    return int(lib().hifa4_cache_page_bytes(int(d)))


def alloc_cache(n_pages, Hkv, d, dtype, device, n_tails) -> PagedCache:
    """Pool of n_pages pages and n_tails tails (one per sequence that grows); dtype: torch.float16 or torch.bfloat16."""
    nb = cache_page_bytes(d)
    if nb == 0:
        raise Hifa4Error(2, "hifa4_cache_page_bytes")
    return PagedCache(torch.zeros((n_pages, Hkv, nb), dtype=torch.uint8, device=device),
                      torch.zeros((n_tails, Hkv, PAGE_TOKENS, d), dtype=dtype, device=device))


# The kernels run on the current device, so every tensor has to be there (get_device() is -1 on the host).  A step of a short dialogue is
# bound by host time: the checks of a call share what they look up.
# A torch without CUDA has neither function: the calls refuse there, the import and the size queries work.
_get_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_I32, _FP32 = torch.int32, torch.float32


def _ok(t, dtype, shape, dev):
    """A contiguous tensor of this type and shape on device `dev`."""
    return t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous()


def _apart(out, q):
    """Whether the caller's output (contiguous) and the queries do not overlap: the CTAs of a call read q at different times."""
    a, b = out.data_ptr(), q.data_ptr()
    return not (a <= b < a + out.nbytes or (q.is_contiguous() and b <= a < b + q.nbytes))


def _seqs(block_table, kv_lens, dev, tail_slots=None) -> _Seqs:
    shape = B, max_pages = block_table.shape
    lens = shape[:1]
    assert _ok(block_table, _I32, shape, dev) and _ok(kv_lens, _I32, lens, dev)
    assert tail_slots is None or _ok(tail_slots, _I32, lens, dev)
    return _Seqs(B, max_pages, block_table.data_ptr(), kv_lens.data_ptr(), None if tail_slots is None else tail_slots.data_ptr())


def _status(t, dev):
    assert t is None or (t.dtype is _I32 and t.get_device() == dev)
    return _ptr(t)


def _strides(t, dev):
    """Reference to the strides of [B,H,n,d] or [B,H,d] (channels contiguous), None where all is contiguous."""
    assert t.get_device() == dev
    if t.is_contiguous():
        return None
    assert t.stride(-1) == 1
    st = [t.stride(i) if t.shape[i] > 1 else 0 for i in range(t.dim() - 1)]
    return C.byref(_Strides(st[0], st[1], st[2] if t.dim() == 4 else 0))


def cache_append(cache: PagedCache, k, v, block_table, kv_lens, n_new=None, inv_s=None, tail_slots=None, d_status=None):
    """Smooths and quantizes new keys and values k, v [B,Hkv,n,d] into the cache's pages.  kv_lens [B] counts the new
    tokens; n_new [B]: how many of the n rows a sequence takes (None: all).  int32 device tensors.
    Before an append a length may be lowered to a multiple of 64, or inside the last page unless that is full and one append
    filled it from its first position on (what v_tail holds: include/hifa4.h)."""
    shape = B, Hkv, n, d = k.shape
    dev, dt = _get_device(), k.dtype
    st, sq = cache.struct(_DT[dt], dev), _seqs(block_table, kv_lens, dev, tail_slots)
    assert v.shape == shape and v.dtype is dt and Hkv == st.Hkv and d == st.d and B == sq.B
    assert cache.v_tail is not None and cache.v_tail.dtype is dt
    assert (n_new is None or _ok(n_new, _I32, shape[:1], dev)) and (inv_s is None or _ok(inv_s, _FP32, (Hkv, d), dev))
    rc = lib().hifa4_cache_append(C.byref(st), C.byref(sq), n, _ptr(n_new), k.data_ptr(), _strides(k, dev), v.data_ptr(),
                                  _strides(v, dev), _ptr(inv_s), _status(d_status, dev), _raw_stream(dev))
    if rc:
        _check(rc, "hifa4_cache_append")


def cache_read(cache: PagedCache, block_table, kv_lens, n, start=None, out_dtype=BF16, out=None, d_status=None):
    """The values in the cache: (k, v) [B,Hkv,n,d], token i of row b at position start[b] + i (None: i).  Rows at or behind
    kv_lens[b] are left as they were in out = (k, v), the caller's tensors, and are zero in new ones."""
    dev = _get_device()
    st, sq = cache.struct(BF16, dev), _seqs(block_table, kv_lens, dev)
    shape = (sq.B, st.Hkv, n, st.d)
    k, v = out if out is not None else [cache.pages.new_zeros(shape, dtype=_TORCH_DT[out_dtype]) for _ in range(2)]
    dt = k.dtype
    assert _ok(k, dt, shape, dev) and _ok(v, dt, shape, dev) and (start is None or _ok(start, _I32, shape[:1], dev))
    rc = lib().hifa4_cache_read(C.byref(st), C.byref(sq), n, _ptr(start), _DT[dt], k.data_ptr(), v.data_ptr(), _status(d_status, dev),
                                _raw_stream(dev))
    if rc:
        _check(rc, "hifa4_cache_read")
    return k, v


@lru_cache(maxsize=1024)
def _cache_workspace_bytes(call, Hkv, d, dtype, B, max_pages, Hq, N, q_to_kv, weight):
    """Size query of "decode" or "attention" by the sizes alone."""
    keep, mp = _map_arr(q_to_kv)
    prm = C.byref(_CacheQuery(Hq, mp, N, 0, F32, 0.0))
    st = C.byref(_Cache(Hkv, d, dtype, 1, None, 0, None))
    if call == "decode":
        return int(lib().hifa4_cache_decode_workspace_bytes(st, B, max_pages, prm, int(weight)))
    return int(lib().hifa4_cache_attention_workspace_bytes(st, B, max_pages, prm))


def _tuple(q_to_kv):
    return None if q_to_kv is None else tuple(int(x) for x in q_to_kv)


def cache_decode_workspace_bytes(cache: PagedCache, B, max_pages, Hq, q_to_kv=None, with_page_weight=False) -> int:
    st = cache.struct(BF16)
    return _cache_workspace_bytes("decode", st.Hkv, st.d, BF16, B, max_pages, Hq, 1, _tuple(q_to_kv), bool(with_page_weight))


def cache_decode(q, cache: PagedCache, block_table, kv_lens, s=None, out=None, lse=None, page_weight=None,
                 page_weight_out=None, workspace=None, softmax_scale=0.0, q_to_kv=None, d_status=None):
    """Attention of one new token per sequence, q [B,Hq,d], over the cache -> out [B,Hq,d] (dtype of `out`, or of q).
    lse [B,Hq], page_weight and page_weight_out [B,max_pages]: float32 device tensors, see include/hifa4.h."""
    q_shape = B, Hq, d = q.shape
    dev, dt, shape = _get_device(), _DT[q.dtype], block_table.shape
    st, sq = cache.struct(dt, dev), _seqs(block_table, kv_lens, dev)
    assert d == st.d and B == sq.B and (s is None or _ok(s, _FP32, (st.Hkv, d), dev)) and (lse is None or _ok(lse, _FP32, (B, Hq), dev))
    assert page_weight is None or _ok(page_weight, _FP32, shape, dev)
    assert page_weight_out is None or _ok(page_weight_out, _FP32, shape, dev)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        assert _ok(out, out.dtype, q_shape, dev) and _apart(out, q)
    if q_to_kv is not None:
        q_to_kv = _tuple(q_to_kv)
    if workspace is None:
        workspace = q.new_empty(_cache_workspace_bytes("decode", st.Hkv, d, dt, B, sq.max_pages, Hq, 1, q_to_kv,
                                                       page_weight_out is not None), dtype=torch.uint8)
    else:
        assert workspace.get_device() == dev
    keep, mp = _map_arr(q_to_kv)
    rc = lib().hifa4_cache_decode(C.byref(st), C.byref(sq), C.byref(_CacheQuery(Hq, mp, 1, 0, _DT[out.dtype], softmax_scale)),
                                  q.data_ptr(), _strides(q, dev), _ptr(s), out.data_ptr(), _ptr(lse), _ptr(page_weight),
                                  _ptr(page_weight_out), workspace.data_ptr(), workspace.nbytes, _status(d_status, dev), _raw_stream(dev))
    if rc:
        _check(rc, "hifa4_cache_decode")
    return out


def cache_attention_workspace_bytes(cache: PagedCache, B, max_pages, Hq, N, dtype=torch.bfloat16, q_to_kv=None) -> int:
    dt = _DT[dtype]
    st = cache.struct(dt)
    return _cache_workspace_bytes("attention", st.Hkv, st.d, dt, B, max_pages, Hq, N, _tuple(q_to_kv), False)


def cache_attention(q, cache: PagedCache, block_table, kv_lens, causal, s=None, out=None, workspace=None, softmax_scale=0.0,
                    q_to_kv=None, d_status=None):
    """Attention of q [B,Hq,N,d] over the cache: all keys of each sequence (cross attention), or, causal, those up to the
    query's own position when the N queries are the sequence's last N tokens -> out [B,Hq,N,d]."""
    q_shape = B, Hq, N, d = q.shape
    dev, dt = _get_device(), _DT[q.dtype]
    st, sq = cache.struct(dt, dev), _seqs(block_table, kv_lens, dev)
    assert d == st.d and B == sq.B and (s is None or _ok(s, _FP32, (st.Hkv, d), dev))
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    else:
        assert _ok(out, out.dtype, q_shape, dev) and _apart(out, q)
    if q_to_kv is not None:
        q_to_kv = _tuple(q_to_kv)
    if workspace is None:
        workspace = q.new_empty(_cache_workspace_bytes("attention", st.Hkv, d, dt, B, sq.max_pages, Hq, N, q_to_kv, False),
                                dtype=torch.uint8)
    else:
        assert workspace.get_device() == dev
    keep, mp = _map_arr(q_to_kv)
    rc = lib().hifa4_cache_attention(C.byref(st), C.byref(sq), C.byref(_CacheQuery(Hq, mp, N, causal, _DT[out.dtype], softmax_scale)),
                                     q.data_ptr(), _strides(q, dev), _ptr(s), out.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                     _status(d_status, dev), _raw_stream(dev))
    if rc:
        _check(rc, "hifa4_cache_attention")
    return out


def selftest_cache_wait_timeout(q, cache: PagedCache, block_table, kv_lens, d_status, out, workspace, page_weight_out=None):
    """Launches the self-test instantiation of the kernel that cache_attention (q [B,Hq,N,d]) or cache_decode (q [B,Hq,d]) would
    take, in which a wait for a page runs out (see include/hifa4.h); q, out and workspace as for those calls.  d_status holds
    HIFA4_ERR_TIMEOUT afterwards."""
    q_shape, shape = q.shape, block_table.shape
    dev, N = _get_device(), q_shape[2] if q.dim() == 4 else 1
    st, sq = cache.struct(_DT[q.dtype], dev), _seqs(block_table, kv_lens, dev)
    assert q.is_contiguous() and q.get_device() == dev and q_shape[-1] == st.d and q_shape[0] == sq.B
    assert _ok(out, out.dtype, q_shape, dev) and _apart(out, q) and workspace.get_device() == dev
    assert page_weight_out is None or _ok(page_weight_out, _FP32, shape, dev)
    rc = lib().hifa4_selftest_cache_wait_timeout(C.byref(st), C.byref(sq), C.byref(_CacheQuery(q_shape[1], None, N, 0, _DT[out.dtype], 0.0)),
                                                 q.data_ptr(), out.data_ptr(), _ptr(page_weight_out), workspace.data_ptr(), workspace.nbytes,
                                                 _status(d_status, dev), _raw_stream(dev))
    _check(rc, "hifa4_selftest_cache_wait_timeout")
    return out


@dataclass
class Evicted:
    """What cache_evict returns: the shorter tables, lengths and weights, and the pages that left."""
    block_table: torch.Tensor
    kv_lens: torch.Tensor
    page_weight: torch.Tensor
    freed: torch.Tensor
    n_freed: torch.Tensor


def alloc_evicted(block_table) -> Evicted:
    B = block_table.shape[0]
    ints = lambda *shape: torch.empty(shape, dtype=torch.int32, device=block_table.device)
    return Evicted(ints(*block_table.shape), ints(B), torch.empty(block_table.shape, dtype=torch.float32, device=block_table.device),
                   ints(*block_table.shape), ints(B))


def cache_evict(block_table, kv_lens, page_weight, keep_pages, keep_first=1, keep_last=1, out: Evicted | None = None,
                d_status=None) -> Evicted:
    """Takes the pages with the least weight out of the block tables of sequences longer than keep_pages pages; the first
    keep_first and the last keep_last stay.  The tensors of `out` may be the inputs."""
    dev, shape = _get_device(), block_table.shape
    lens = shape[:1]
    sq = _seqs(block_table, kv_lens, dev)
    if out is None:
        out = alloc_evicted(block_table)
    assert _ok(page_weight, _FP32, shape, dev) and _ok(out.block_table, _I32, shape, dev) and _ok(out.kv_lens, _I32, lens, dev)
    assert _ok(out.page_weight, _FP32, shape, dev) and _ok(out.freed, _I32, shape, dev) and _ok(out.n_freed, _I32, lens, dev)
    rc = lib().hifa4_cache_evict(C.byref(sq), page_weight.data_ptr(), keep_pages, keep_first, keep_last, out.block_table.data_ptr(),
                                 out.kv_lens.data_ptr(), out.page_weight.data_ptr(), out.freed.data_ptr(), out.n_freed.data_ptr(),
                                 _status(d_status, dev), _raw_stream(dev))
    if rc:
        _check(rc, "hifa4_cache_evict")
    return out
