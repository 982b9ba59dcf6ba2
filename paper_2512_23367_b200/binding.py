"""ctypes binding of libpq.so.  Marshals torch CUDA tensors (device pointers, sizes, the current
stream) into the C calls of ``include/pq.h``; every step of the computation runs in the library's
kernels.  torch is used for device memory and streams only."""
from __future__ import annotations

import ctypes
import os

import torch

from . import build as _build

GROUP = 128

_lib = None

_i64, _i32, _vp, _f64 = ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p, ctypes.c_double

# name -> (restype, argtypes); mirrors include/pq.h
SIGNATURES = {
    "pq_status_str": (ctypes.c_char_p, [ctypes.c_int]),
    "pq_last_cuda_error": (ctypes.c_char_p, []),
    "pq_packed_w8_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "pq_packed_w4_bytes": (ctypes.c_size_t, [_i64, _i64]),
    "pq_quantize_act": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w8": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w4": (ctypes.c_int, [_vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "pq_unpack_w8": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp]),
    "pq_unpack_w4": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp]),
    "pq_gemm_w8a8": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, ctypes.c_size_t, _vp]),
    "pq_gemm_w4a8": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i32, _i64, _i64, _i64, _vp, _vp]),
    "pq_acc_w8a8": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i64, _vp, _vp]),
    "pq_acc_w4a8": (ctypes.c_int, [_vp, _vp, _i32, _i64, _i64, _i64, _vp, _vp]),
    "pq_device_status": (ctypes.c_int, [ctypes.POINTER(ctypes.c_int)]),
    "pq_workspace_bytes": (ctypes.c_size_t, [_i64, ctypes.POINTER(_i64), _i32, _i64, _i32]),
    "pq_workspace_init": (ctypes.c_int, [_vp, ctypes.c_size_t, _vp]),
    "pq_set_wait_limit": (ctypes.c_int, [ctypes.c_uint32]),
    "pq_plan_w8a8": (ctypes.c_int, [_i64, _i64, _i64, _i32, ctypes.c_size_t, ctypes.POINTER(_i32), ctypes.POINTER(_i32)]),
    "pq_gemm_w8a8_noalloc": (ctypes.c_int, [_vp, _vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp]),
    "pq_gemm_w8a8_group": (ctypes.c_int, [_vp, _vp, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp),
                                          ctypes.POINTER(_i64), ctypes.POINTER(_vp), _i64, _i64, _vp,
                                          ctypes.c_size_t, _vp]),
    "pq_quantize_act_static": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_swiglu_quantize": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_linear_w8a8": (ctypes.c_int, [_vp, _vp, _vp, _i64, _i64, _i64, _vp, _vp, _vp, _vp, ctypes.c_size_t, _vp]),
    "pq_linear_w4a8": (ctypes.c_int, [_vp, _vp, _vp, _i32, _i64, _i64, _i64, _vp, _vp, _vp, _vp]),
    "pq_quantize_act_static_channel": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_hadamard_block": (_i32, [_i64]),
    "pq_quantize_act_hadamard": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w8_hadamard": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w4_hadamard": (ctypes.c_int, [_vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "pq_col_absmax": (ctypes.c_int, [_vp, _i64, _i64, _vp, _vp]),
    "pq_smooth_scales": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _vp]),
    "pq_smooth_scales_alpha": (ctypes.c_int, [_vp, _vp, _i64, _i32, _vp, _vp, _vp]),
    "pq_quantize_act_smooth": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w8_smooth": (ctypes.c_int, [_vp, _vp, _i64, _i64, _vp, _vp, _vp]),
    "pq_pack_w4_smooth": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "pq_gemm_w4a8_group": (ctypes.c_int, [_vp, _vp, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_vp), _i32,
                                          ctypes.POINTER(_i64), ctypes.POINTER(_vp), _i64, _i64, _vp]),
    "pq_block_tables": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i32, _i64, _vp, _vp, _vp, _vp, _vp, _vp]),
    "pq_kv_append": (ctypes.c_int, [_vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp]),
    "pq_kv_read": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _vp]),
    "pq_paged_attention": (ctypes.c_int, [_vp, _i64, _i32, _vp, _vp, _i64, _vp, _vp, _i64, _i64, _i64, _i64,
                                          ctypes.c_float, _i32, _vp, _vp, ctypes.c_size_t, _vp]),
    "pq_attention_workspace_bytes": (ctypes.c_size_t, [_i64, _i64, _i64, _i64, _i32, _i32, _i32, _i32]),
    "pq_rotary_frequencies": (ctypes.c_int, [_i32, _f64, _i32, _f64, _f64, _f64, _f64, _vp, _vp]),
    "pq_rotate": (ctypes.c_int, [_vp, _vp, _i64, _i64, _i32, _i32, _vp, _i64, _vp, _i64, _i64, _vp]),
    "pq_kv_append_rotated": (ctypes.c_int, [_vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _i64, _i32, _vp, _i64, _i64, _vp]),
    "pq_latent_append": (ctypes.c_int, [_vp, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _i64, _i32, _vp, _i64, _i64, _vp]),
    "pq_latent_read": (ctypes.c_int, [_vp, _vp, _i64, _vp, _vp, _vp]),
    "pq_head_linear": (ctypes.c_int, [_vp, _i64, _i64, _vp, _i32, _i64, _i64, _i64, _vp, _i64, _i64, _vp]),
    "pq_latent_attention": (ctypes.c_int, [_vp, _i32, _vp, _vp, _i64, _vp, _vp, _i64, _i64, ctypes.c_float, _vp, _vp,
                                           ctypes.c_size_t, _vp]),
    "pq_latent_workspace_bytes": (ctypes.c_size_t, [_i32]),
    "pq_expanded_attention": (ctypes.c_int, [_vp, _i64, _i32, _vp, _i64, _vp, _i64, _i64, _vp, _vp, _i64, _i64, _i64,
                                             ctypes.c_float, _vp, _vp, ctypes.c_size_t, _vp]),
    "pq_attention_workspace_bytes_window": (ctypes.c_size_t, [_i64, _i64, _i64, _i64, _i32, _i32, _i32, _i32, _i32]),
}
MAX_GROUP = 4
MAX_REQUESTS = 4096


class PQError(RuntimeError):
    def __init__(self, call: str, status: int):
        self.status = status
        msg = lib().pq_status_str(status).decode() if _lib is not None else "?"
        if status == 5 and _lib is not None:
            msg += ": " + lib().pq_last_cuda_error().decode()
        super().__init__(f"{call} failed: status {status} ({msg})")


def lib() -> ctypes.CDLL:
    """Load (building first if missing or stale) libpq.so.  Raises if that is impossible."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if _build.stale():
            path = _build.build()
        if not os.path.exists(path):
            raise RuntimeError(f"CUDA library {path} is missing and could not be built")
        handle = ctypes.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)  # AttributeError if the library lacks a declared symbol
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


# The current device and its current stream's handle.  torch.cuda.current_stream() builds a Stream object, 3 us of a
# call that takes 7; torch's own launchers read the handle directly, and so does this where torch offers it.
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream if _raw_stream is None else _raw_stream(_device())


def _dev(t: torch.Tensor, dtype: torch.dtype, what: str) -> torch.Tensor:
    if not t.is_cuda:
        raise ValueError(f"{what}: expected a CUDA tensor (this library has no CPU path)")
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    return t


def _check(call: str, status: int) -> None:
    if status != 0:
        raise PQError(call, status)


def _sized(t: torch.Tensor, dtype: torch.dtype, numel: int, what: str) -> torch.Tensor:
    """A contiguous tensor of `dtype` with exactly `numel` elements.  The C calls take raw pointers and trust
    the sizes they are given, so a short buffer would become an out-of-bounds device access: every operand is
    measured here, before anything is launched (and before the devices are looked at, so that a wrong size is
    reported as such wherever the tensor lives)."""
    if t.dtype != dtype:
        raise TypeError(f"{what}: expected {dtype}, got {t.dtype}")
    if t.numel() != int(numel):
        raise ValueError(f"{what}: expected {int(numel)} elements, got {t.numel()}")
    if not t.is_contiguous():
        raise ValueError(f"{what}: expected a contiguous tensor")
    return t


def _together(first: torch.Tensor, *others: torch.Tensor | None) -> None:
    """All operands of a call live on one CUDA device."""
    if not first.is_cuda:
        raise ValueError("expected CUDA tensors (this library has no CPU path)")
    for t in others:
        if t is not None and t.device != first.device:
            raise ValueError(f"operands on different devices: {t.device} and {first.device}")


def _tokens(q: torch.Tensor, s_tok: torch.Tensor) -> tuple[int, int]:
    """Measures the quantized tokens (q int8 [M,K], s_tok f32 [M]); returns (M, K)."""
    if q.dim() != 2:
        raise ValueError("q: expected a 2-D tensor [M,K]")
    M, K = q.shape
    _sized(q, torch.int8, M * K, "q")
    _sized(s_tok, torch.float32, M, "s_tok")
    return int(M), int(K)


def _out(y: torch.Tensor | None, M: int, N: int, like: torch.Tensor) -> torch.Tensor:
    if y is None:
        return torch.empty((M, N), dtype=torch.float16, device=like.device)
    return _sized(y, torch.float16, M * N, "y")


def _ws(workspace: torch.Tensor | None) -> tuple[int | None, int]:
    if workspace is None:
        return None, 0
    _sized(workspace, torch.uint8, workspace.numel(), "workspace")
    return workspace.data_ptr(), workspace.numel()


def _factors(v: torch.Tensor, K: int, name: str) -> torch.Tensor:
    """A per-column factor vector f32 [K] on the device."""
    return _dev(_sized(v, torch.float32, K, name), torch.float32, name)


def _rows(x: torch.Tensor, q: torch.Tensor | None, s_tok: torch.Tensor | None):
    """Outputs of a row quantizer for x f16 [M,K]: created when absent, measured when given."""
    if x.dim() != 2:
        raise ValueError("x: expected a 2-D tensor [M,K]")
    M, K = x.shape
    _sized(x, torch.float16, M * K, "x")
    if q is not None:
        _sized(q, torch.int8, M * K, "q")
    if s_tok is not None:
        _sized(s_tok, torch.float32, M, "s_tok")
    _together(x, q, s_tok)
    q = torch.empty((M, K), dtype=torch.int8, device=x.device) if q is None else q
    s_tok = torch.empty((M,), dtype=torch.float32, device=x.device) if s_tok is None else s_tok
    return int(M), int(K), q, s_tok


def pq_quantize_act(x: torch.Tensor, q: torch.Tensor | None = None, s_tok: torch.Tensor | None = None):
    """x f16 [M,K] -> (q int8 [M,K], s_tok f32 [M])."""
    M, K, q, s_tok = _rows(x, q, s_tok)
    _check("pq_quantize_act", lib().pq_quantize_act(x.data_ptr(), M, K, q.data_ptr(), s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_quantize_act_smooth(x: torch.Tensor, s_inv: torch.Tensor, q: torch.Tensor | None = None,
                           s_tok: torch.Tensor | None = None):
    """Quantizes X S^-1 (Eq. 3): x f16 [M,K], s_inv f32 [K] -> (q int8 [M,K], s_tok f32 [M])."""
    M, K, q, s_tok = _rows(x, q, s_tok)
    s_inv = _factors(s_inv, K, "s_inv")
    _check("pq_quantize_act_smooth", lib().pq_quantize_act_smooth(x.data_ptr(), s_inv.data_ptr(), M, K, q.data_ptr(),
                                                                  s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_quantize_act_static(x: torch.Tensor, scale: torch.Tensor, q: torch.Tensor | None = None,
                           s_tok: torch.Tensor | None = None):
    """INT8 codes against one calibrated scale: x f16 [M,K], scale f32 device tensor with one element
    -> (q int8 [M,K], s_tok f32 [M] filled with the scale)."""
    M, K, q, s_tok = _rows(x, q, s_tok)
    scale = _sized(scale, torch.float32, 1, "scale")
    _together(x, scale)
    _check("pq_quantize_act_static", lib().pq_quantize_act_static(x.data_ptr(), scale.data_ptr(), M, K, q.data_ptr(),
                                                                  s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_quantize_act_static_channel(x: torch.Tensor, inv_s: torch.Tensor, q: torch.Tensor | None = None,
                                   s_tok: torch.Tensor | None = None):
    """INT8 codes against one calibrated scale per feature channel: x f16 [M,K], inv_s f32 [K] (reciprocal
    scales) -> (q int8 [M,K], s_tok f32 [M] = 1; fold the channel scales into the weights)."""
    M, K, q, s_tok = _rows(x, q, s_tok)
    inv_s = _factors(inv_s, K, "inv_s")
    _together(x, inv_s)
    _check("pq_quantize_act_static_channel", lib().pq_quantize_act_static_channel(x.data_ptr(), inv_s.data_ptr(), M, K,
                                                                                  q.data_ptr(), s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_swiglu_quantize(gate: torch.Tensor, up: torch.Tensor, q: torch.Tensor | None = None,
                       s_tok: torch.Tensor | None = None):
    """The MLP's gated activation fused with the down projection's quantizer: gate, up f16 [M,I] ->
    (q int8 [M,I], s_tok f32 [M]) of h = silu(gate) * up."""
    M, I, q, s_tok = _rows(gate, q, s_tok)
    _sized(up, torch.float16, M * I, "up")
    _together(gate, up)
    _check("pq_swiglu_quantize", lib().pq_swiglu_quantize(gate.data_ptr(), up.data_ptr(), M, I, q.data_ptr(),
                                                          s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_hadamard_block(K: int) -> int:
    """Order of the Hadamard blocks the Eq. 4 calls use for rows of length K (host-only query)."""
    return int(lib().pq_hadamard_block(int(K)))


def pq_quantize_act_hadamard(x: torch.Tensor, q: torch.Tensor | None = None, s_tok: torch.Tensor | None = None):
    """Quantizes X H (Eq. 4): x f16 [M,K] -> (q int8 [M,K], s_tok f32 [M])."""
    M, K, q, s_tok = _rows(x, q, s_tok)
    _check("pq_quantize_act_hadamard", lib().pq_quantize_act_hadamard(x.data_ptr(), M, K, q.data_ptr(),
                                                                      s_tok.data_ptr(), _stream()))
    return q, s_tok


def pq_pack_w8_hadamard(w: torch.Tensor):
    """Packs W H (Eq. 4): w f16 [N,K] -> (wq opaque uint8 buffer, s_ch f32 [N])."""
    w = _dev(w, torch.float16, "w")
    N, K = w.shape
    wq = torch.empty((lib().pq_packed_w8_bytes(N, K),), dtype=torch.uint8, device=w.device)
    s_ch = torch.empty((N,), dtype=torch.float32, device=w.device)
    _check("pq_pack_w8_hadamard", lib().pq_pack_w8_hadamard(w.data_ptr(), N, K, wq.data_ptr(), s_ch.data_ptr(), _stream()))
    return wq, s_ch


def pq_pack_w4_hadamard(w: torch.Tensor, group: int = GROUP):
    """Packs W H (Eq. 4): w f16 [N,K] -> (wp opaque uint8 buffer, s_grp f16 [K/group, N])."""
    w = _dev(w, torch.float16, "w")
    N, K = w.shape
    wp = torch.empty((lib().pq_packed_w4_bytes(N, K),), dtype=torch.uint8, device=w.device)
    s_grp = torch.empty((max(K // max(group, 1), 1), N), dtype=torch.float16, device=w.device)
    _check("pq_pack_w4_hadamard", lib().pq_pack_w4_hadamard(w.data_ptr(), N, K, group, wp.data_ptr(), s_grp.data_ptr(),
                                                            _stream()))
    return wp, s_grp


def pq_col_absmax(a: torch.Tensor) -> torch.Tensor:
    """a f16 [R,K] -> f32 [K]: column maxima of |a| (calibration statistic of Eq. 3)."""
    a = _dev(a, torch.float16, "a")
    R, K = a.shape
    out = torch.empty((K,), dtype=torch.float32, device=a.device)
    _check("pq_col_absmax", lib().pq_col_absmax(a.data_ptr(), R, K, out.data_ptr(), _stream()))
    return out


def pq_smooth_scales(x_absmax: torch.Tensor, w_absmax: torch.Tensor, alpha_quarters: int = 2):
    """Eq. 3: (s, s_inv) f32 [K] from the column maxima of X and of W, alpha = alpha_quarters / 4 (default 1/2)."""
    xa = _dev(x_absmax, torch.float32, "x_absmax")
    wa = _factors(w_absmax, xa.shape[0], "w_absmax")
    s, s_inv = torch.empty_like(xa), torch.empty_like(xa)
    _check("pq_smooth_scales_alpha", lib().pq_smooth_scales_alpha(xa.data_ptr(), wa.data_ptr(), xa.shape[0],
                                                                  int(alpha_quarters), s.data_ptr(), s_inv.data_ptr(),
                                                                  _stream()))
    return s, s_inv


def pq_pack_w8(w: torch.Tensor, smooth: torch.Tensor | None = None):
    """w f16 [N,K] -> (wq opaque uint8 buffer, s_ch f32 [N]).  With smooth f32 [K]: packs S W (Eq. 3)."""
    w = _dev(w, torch.float16, "w")
    N, K = w.shape
    wq = torch.empty((lib().pq_packed_w8_bytes(N, K),), dtype=torch.uint8, device=w.device)
    s_ch = torch.empty((N,), dtype=torch.float32, device=w.device)
    if smooth is None:
        _check("pq_pack_w8", lib().pq_pack_w8(w.data_ptr(), N, K, wq.data_ptr(), s_ch.data_ptr(), _stream()))
    else:
        smooth = _factors(smooth, K, "smooth")
        _check("pq_pack_w8_smooth", lib().pq_pack_w8_smooth(w.data_ptr(), smooth.data_ptr(), N, K, wq.data_ptr(),
                                                            s_ch.data_ptr(), _stream()))
    return wq, s_ch


def pq_pack_w4(w: torch.Tensor, group: int = GROUP, smooth: torch.Tensor | None = None):
    """w f16 [N,K] -> (wp opaque uint8 buffer, s_grp f16 [K/group, N]).  With smooth f32 [K]: packs S W (Eq. 3)."""
    w = _dev(w, torch.float16, "w")
    N, K = w.shape
    wp = torch.empty((lib().pq_packed_w4_bytes(N, K),), dtype=torch.uint8, device=w.device)
    s_grp = torch.empty((max(K // max(group, 1), 1), N), dtype=torch.float16, device=w.device)
    if smooth is None:
        _check("pq_pack_w4", lib().pq_pack_w4(w.data_ptr(), N, K, group, wp.data_ptr(), s_grp.data_ptr(), _stream()))
    else:
        smooth = _factors(smooth, K, "smooth")
        _check("pq_pack_w4_smooth", lib().pq_pack_w4_smooth(w.data_ptr(), smooth.data_ptr(), N, K, group, wp.data_ptr(),
                                                            s_grp.data_ptr(), _stream()))
    return wp, s_grp


def pq_unpack_w8(wq: torch.Tensor, N: int, K: int) -> torch.Tensor:
    wq = _dev(_sized(wq, torch.uint8, N * K, "wq"), torch.uint8, "wq")
    codes = torch.empty((N, K), dtype=torch.int8, device=wq.device)
    _check("pq_unpack_w8", lib().pq_unpack_w8(wq.data_ptr(), N, K, codes.data_ptr(), _stream()))
    return codes


def pq_unpack_w4(wp: torch.Tensor, N: int, K: int) -> torch.Tensor:
    wp = _dev(_sized(wp, torch.uint8, N * K // 2, "wp"), torch.uint8, "wp")
    codes = torch.empty((N, K), dtype=torch.int8, device=wp.device)
    _check("pq_unpack_w4", lib().pq_unpack_w4(wp.data_ptr(), N, K, codes.data_ptr(), _stream()))
    return codes


def pq_plan_w8a8(M: int, N: int, K: int, sms: int = 148, scratch_bytes: int = 0) -> tuple[int, int]:
    """(tile width, number of K parts) the W8A8 GEMM would choose; host-only, needs no GPU."""
    bn, sp = _i32(0), _i32(0)
    _check("pq_plan_w8a8", lib().pq_plan_w8a8(M, N, K, sms, scratch_bytes, ctypes.byref(bn), ctypes.byref(sp)))
    return int(bn.value), int(sp.value)


def pq_workspace_bytes(M: int, Ns, K: int, sms: int = 148) -> int:
    """Bytes of workspace with which pq_gemm_w8a8 (Ns = one width) or pq_gemm_w8a8_group (Ns = the members'
    widths) at these M and K runs the schedule it would pick with unlimited room; 0 if that schedule does not
    split K.  Host-only, needs no GPU."""
    Ns = [int(Ns)] if isinstance(Ns, int) else [int(n) for n in Ns]
    arr = (_i64 * max(len(Ns), 1))(*Ns)
    return int(lib().pq_workspace_bytes(int(M), arr, len(Ns), int(K), int(sms)))


def pq_workspace_init(workspace: torch.Tensor) -> torch.Tensor:
    """Prepares a caller-owned workspace (uint8 CUDA tensor, 256-byte aligned, >= 64 KiB) for the W8A8 calls
    on the current stream: zeroes its arrival counters.  Returns the tensor."""
    workspace = _dev(workspace, torch.uint8, "workspace")
    with torch.cuda.device(workspace.device):
        _check("pq_workspace_init", lib().pq_workspace_init(workspace.data_ptr(), workspace.numel(), _stream()))
    return workspace


def pq_set_wait_limit(polls: int) -> None:
    """Poll bound of the waits inside kernels launched from now on (0 = the default).  Test hook."""
    _check("pq_set_wait_limit", lib().pq_set_wait_limit(int(polls)))


def pq_gemm_w8a8(q, s_tok, wq, s_ch, N: int, y: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None) -> torch.Tensor:
    """q int8 [M,K], s_tok f32 [M], wq/s_ch from pq_pack_w8 -> y f16 [M,N].  workspace: optional prepared
    scratch of this call (pq_workspace_bytes / pq_workspace_init); without it K is never split."""
    M, K = _tokens(q, s_tok)
    _sized(wq, torch.uint8, N * K, "wq"), _sized(s_ch, torch.float32, N, "s_ch")
    ws, ws_bytes = _ws(workspace)
    if y is not None:
        _sized(y, torch.float16, M * N, "y")
    _together(q, s_tok, wq, s_ch, y, workspace)
    y = _out(y, M, N, q)
    _check("pq_gemm_w8a8", lib().pq_gemm_w8a8(q.data_ptr(), s_tok.data_ptr(), wq.data_ptr(), s_ch.data_ptr(),
                                              M, N, K, y.data_ptr(), ws, ws_bytes, _stream()))
    return y


def _group_arrays(q, s_tok, members, ys, w_dtype, w_numel, s_dtype, s_numel, M, workspace=None):
    n = len(members)
    if not 1 <= n <= MAX_GROUP:
        raise ValueError(f"a group holds 1..{MAX_GROUP} members")
    if ys is None:
        ys = [None] * n
    if len(ys) != n:
        raise ValueError("one output per member")
    for i, ((w, sc, N), y) in enumerate(zip(members, ys)):
        N = int(N)
        _sized(w, w_dtype, w_numel(N), f"members[{i}] weights")
        _sized(sc, s_dtype, s_numel(N), f"members[{i}] scales")
        if y is not None:
            _sized(y, torch.float16, M * N, f"ys[{i}]")
    _together(q, s_tok, workspace, *[m[0] for m in members], *[m[1] for m in members], *ys)
    outs = [_out(y, M, int(m[2]), q) for m, y in zip(members, ys)]
    w_arr = (_vp * n)(*[m[0].data_ptr() for m in members])
    s_arr = (_vp * n)(*[m[1].data_ptr() for m in members])
    n_arr = (_i64 * n)(*[int(m[2]) for m in members])
    y_arr = (_vp * n)(*[y.data_ptr() for y in outs])
    return n, w_arr, s_arr, n_arr, y_arr, outs


def pq_gemm_w8a8_group(q, s_tok, members, ys=None, workspace: torch.Tensor | None = None) -> list[torch.Tensor]:
    """Several W8A8 linears over the same quantized tokens as one call (one kernel launch).  members: sequence of (wq, s_ch, N) from pq_pack_w8; ys: optional outputs f16 [M,N_g]; workspace: as for pq_gemm_w8a8.
    Returns the outputs; each equals pq_gemm_w8a8(q, s_tok, wq, s_ch, N) bit for bit."""
    M, K = _tokens(q, s_tok)
    ws, ws_bytes = _ws(workspace)
    n, wq_arr, sc_arr, n_arr, y_arr, outs = _group_arrays(q, s_tok, members, ys, torch.uint8, lambda N: N * K,
                                                          torch.float32, lambda N: N, M, workspace)
    _check("pq_gemm_w8a8_group", lib().pq_gemm_w8a8_group(q.data_ptr(), s_tok.data_ptr(), n, wq_arr, sc_arr, n_arr,
                                                          y_arr, M, K, ws, ws_bytes, _stream()))
    return outs


def pq_gemm_w4a8_group(q, s_tok, members, ys=None, group: int = GROUP) -> list[torch.Tensor]:
    """Several W4A8 linears over the same quantized tokens as one call (one kernel launch).  members: sequence of (wp, s_grp, N) from pq_pack_w4; ys: optional outputs f16 [M,N_g].
    Each output equals pq_gemm_w4a8(q, s_tok, wp, s_grp, N) bit for bit."""
    M, K = _tokens(q, s_tok)
    n, wp_arr, sg_arr, n_arr, y_arr, outs = _group_arrays(q, s_tok, members, ys, torch.uint8, lambda N: N * K // 2,
                                                          torch.float16, lambda N: (K // max(group, 1)) * N, M)
    _check("pq_gemm_w4a8_group", lib().pq_gemm_w4a8_group(q.data_ptr(), s_tok.data_ptr(), n, wp_arr, sg_arr, group,
                                                          n_arr, y_arr, M, K, _stream()))
    return outs


def pq_gemm_w8a8_noalloc(q, s_tok, wq, s_ch, N: int, y: torch.Tensor) -> torch.Tensor:
    """Same product as pq_gemm_w8a8, for callers that may not allocate: the output tensor is
    required (this wrapper creates none) and the library's built-in scratch array is used instead of
    a workspace.  Raises PQError with status 7 when M > 128 and the padded output exceeds 2 Mi
    elements.  Calls on one device must not overlap on the GPU."""
    M, K = _tokens(q, s_tok)
    _sized(wq, torch.uint8, N * K, "wq"), _sized(s_ch, torch.float32, N, "s_ch")
    if y is None:
        raise ValueError("y: required (this entry point creates no tensor)")
    _sized(y, torch.float16, M * N, "y")
    _together(q, s_tok, wq, s_ch, y)
    _check("pq_gemm_w8a8_noalloc", lib().pq_gemm_w8a8_noalloc(q.data_ptr(), s_tok.data_ptr(), wq.data_ptr(),
                                                              s_ch.data_ptr(), M, N, K, y.data_ptr(), _stream()))
    return y


def pq_gemm_w4a8(q, s_tok, wp, s_grp, N: int, group: int = GROUP, y: torch.Tensor | None = None) -> torch.Tensor:
    """q int8 [M,K], s_tok f32 [M], wp/s_grp from pq_pack_w4 -> y f16 [M,N]."""
    M, K = _tokens(q, s_tok)
    _sized(wp, torch.uint8, N * K // 2, "wp"), _sized(s_grp, torch.float16, (K // max(group, 1)) * N, "s_grp")
    if y is not None:
        _sized(y, torch.float16, M * N, "y")
    _together(q, s_tok, wp, s_grp, y)
    y = _out(y, M, N, q)
    _check("pq_gemm_w4a8", lib().pq_gemm_w4a8(q.data_ptr(), s_tok.data_ptr(), wp.data_ptr(), s_grp.data_ptr(),
                                              group, M, N, K, y.data_ptr(), _stream()))
    return y


def _linear_args(x, y, q_tmp, s_tok_tmp, N):
    if x.dim() != 2:
        raise ValueError("x: expected a 2-D tensor [M,K]")
    M, K = x.shape
    _sized(x, torch.float16, M * K, "x")
    if q_tmp is None:
        q_tmp = torch.empty((M, K), dtype=torch.int8, device=x.device)
    if s_tok_tmp is None:
        s_tok_tmp = torch.empty((M,), dtype=torch.float32, device=x.device)
    _sized(q_tmp, torch.int8, M * K, "q_tmp"), _sized(s_tok_tmp, torch.float32, M, "s_tok_tmp")
    if y is not None:
        _sized(y, torch.float16, M * N, "y")
    return M, K, _out(y, M, N, x), q_tmp, s_tok_tmp


def pq_linear_w8a8(x, wq, s_ch, N: int, y: torch.Tensor | None = None, q_tmp: torch.Tensor | None = None,
                   s_tok_tmp: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """x f16 [M,K] -> y f16 [M,N]: pq_quantize_act + pq_gemm_w8a8 in one call (one launch for one to four tokens
    where the row kernel serves).  q_tmp / s_tok_tmp: the caller's buffers for codes and scales (allocated here
    when not given)."""
    M, K, y, q_tmp, s_tok_tmp = _linear_args(x, y, q_tmp, s_tok_tmp, N)
    _sized(wq, torch.uint8, N * K, "wq"), _sized(s_ch, torch.float32, N, "s_ch")
    ws, ws_bytes = _ws(workspace)
    _together(x, wq, s_ch, y, q_tmp, s_tok_tmp, workspace)
    _check("pq_linear_w8a8", lib().pq_linear_w8a8(x.data_ptr(), wq.data_ptr(), s_ch.data_ptr(), M, N, K, y.data_ptr(),
                                                  q_tmp.data_ptr(), s_tok_tmp.data_ptr(), ws, ws_bytes, _stream()))
    return y


def pq_linear_w4a8(x, wp, s_grp, N: int, group: int = GROUP, y: torch.Tensor | None = None,
                   q_tmp: torch.Tensor | None = None, s_tok_tmp: torch.Tensor | None = None) -> torch.Tensor:
    """x f16 [M,K] -> y f16 [M,N]: pq_quantize_act + pq_gemm_w4a8 in one call (see pq_linear_w8a8)."""
    M, K, y, q_tmp, s_tok_tmp = _linear_args(x, y, q_tmp, s_tok_tmp, N)
    _sized(wp, torch.uint8, N * K // 2, "wp"), _sized(s_grp, torch.float16, (K // max(group, 1)) * N, "s_grp")
    _together(x, wp, s_grp, y, q_tmp, s_tok_tmp)
    _check("pq_linear_w4a8", lib().pq_linear_w4a8(x.data_ptr(), wp.data_ptr(), s_grp.data_ptr(), group, M, N, K,
                                                  y.data_ptr(), q_tmp.data_ptr(), s_tok_tmp.data_ptr(), _stream()))
    return y


def pq_acc_w8a8(q, wq, N: int) -> torch.Tensor:
    """Exact INT32 accumulators [M,N] of the W8A8 product."""
    if q.dim() != 2:
        raise ValueError("q: expected a 2-D tensor [M,K]")
    M, K = q.shape
    _sized(q, torch.int8, M * K, "q"), _sized(wq, torch.uint8, N * K, "wq")
    _together(q, wq)
    acc = torch.empty((M, N), dtype=torch.int32, device=q.device)
    _check("pq_acc_w8a8", lib().pq_acc_w8a8(q.data_ptr(), wq.data_ptr(), M, N, K, acc.data_ptr(), _stream()))
    return acc


def pq_acc_w4a8(q, wp, N: int, group: int = GROUP) -> torch.Tensor:
    """Exact INT32 per-group accumulators [K/group, M, N] of the W4A8 product."""
    if q.dim() != 2:
        raise ValueError("q: expected a 2-D tensor [M,K]")
    M, K = q.shape
    _sized(q, torch.int8, M * K, "q"), _sized(wp, torch.uint8, N * K // 2, "wp")
    _together(q, wp)
    acc = torch.empty((K // group, M, N), dtype=torch.int32, device=q.device)
    _check("pq_acc_w4a8", lib().pq_acc_w4a8(q.data_ptr(), wp.data_ptr(), group, M, N, K, acc.data_ptr(), _stream()))
    return acc


# ---- paged key/value cache and attention over it ---------------------------------------------------------

class _KVCache(ctypes.Structure):   # pq_kv_cache of include/pq.h
    _fields_ = [("k", _vp), ("v", _vp), ("k_scale", _vp), ("v_scale", _vp), ("pages", _i64), ("heads", _i32),
                ("page", _i32), ("dim", _i32), ("type", _i32)]


class PagedKV:
    """A paged key/value cache: k, v f16 or int8 [pages, heads, page, dim], for int8 with k_scale, v_scale
    f32 [pages, heads, page].  Measures its tensors once and keeps them; page a multiple of 16, dim 64 or 128."""

    __slots__ = ("k", "v", "k_scale", "v_scale", "pages", "heads", "page", "dim", "device", "_struct", "_ref")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None):
        if k.dim() != 4:
            raise ValueError("k: expected a 4-D tensor [pages, heads, page, dim]")
        pages, heads, page, dim = k.shape
        if k.dtype not in (torch.float16, torch.int8):
            raise TypeError(f"k: expected torch.float16 or torch.int8, got {k.dtype}")
        int8 = k.dtype == torch.int8
        _sized(k, k.dtype, k.numel(), "k"), _sized(v, k.dtype, k.numel(), "v")
        if v.shape != k.shape:
            raise ValueError(f"v: expected the shape of k {tuple(k.shape)}, got {tuple(v.shape)}")
        for s, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if int8 != (s is not None):
                raise ValueError(f"{name}: {'required for an int8 cache' if int8 else 'an f16 cache has none'}")
            if s is not None:
                _sized(s, torch.float32, pages * heads * page, name)
        _together(k, v, k_scale, v_scale)
        put = object.__setattr__
        put(self, "k", k), put(self, "v", v), put(self, "k_scale", k_scale), put(self, "v_scale", v_scale)
        put(self, "pages", pages), put(self, "heads", heads), put(self, "page", page), put(self, "dim", dim)
        put(self, "device", k.get_device())
        put(self, "_struct", _KVCache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if int8 else None,
                                      v_scale.data_ptr() if int8 else None, pages, heads, page, dim, int(int8)))
        put(self, "_ref", ctypes.addressof(self._struct))

    def __setattr__(self, name, value):
        raise AttributeError("a PagedKV is fixed; make another one over other tensors")

    @classmethod
    def empty(cls, pages: int, heads: int, page: int, dim: int, dtype: torch.dtype = torch.float16, device="cuda"):
        """A zero-filled cache."""
        k, v = (torch.zeros((pages, heads, page, dim), dtype=dtype, device=device) for _ in range(2))
        if dtype != torch.int8:
            return cls(k, v)
        return cls(k, v, *(torch.zeros((pages, heads, page), dtype=torch.float32, device=device) for _ in range(2)))


class PagedStep:
    """What pq_block_tables gives for one step: row ranges, cached tokens with the new ones, slots and positions of
    the new tokens, and the head of the free list after the step.  Measures its tensors once and keeps them."""

    __slots__ = ("q_start", "kv_len", "slots", "pos", "free_head", "requests", "tokens", "device", "_ptrs")

    def __init__(self, q_start: torch.Tensor, kv_len: torch.Tensor, slots: torch.Tensor, pos: torch.Tensor,
                 free_head: torch.Tensor):
        B, T = kv_len.numel(), slots.numel()
        _sized(q_start, torch.int32, B + 1, "q_start"), _sized(kv_len, torch.int32, B, "kv_len")
        _sized(slots, torch.int64, T, "slots"), _sized(pos, torch.int32, T, "pos")
        _sized(free_head, torch.int32, 1, "free_head")
        _together(q_start, kv_len, slots, pos, free_head)
        put = object.__setattr__
        put(self, "q_start", q_start), put(self, "kv_len", kv_len), put(self, "slots", slots), put(self, "pos", pos)
        put(self, "free_head", free_head), put(self, "requests", B), put(self, "tokens", T)
        put(self, "device", q_start.get_device())
        put(self, "_ptrs", tuple(x.data_ptr() for x in (q_start, kv_len, slots, pos, free_head)))

    def __setattr__(self, name, value):
        raise AttributeError("a PagedStep is fixed; make another one over other tensors")

    @classmethod
    def empty(cls, requests: int, tokens: int, device="cuda"):
        """Buffers for a step of up to `tokens` new tokens."""
        i32 = lambda n: torch.empty((n,), dtype=torch.int32, device=device)  # noqa: E731
        return cls(i32(requests + 1), i32(requests), torch.empty((tokens,), dtype=torch.int64, device=device),
                   i32(tokens), i32(1))


def _operands(device: int, *checks) -> None:
    """(tensor, dtype, elements, name) of every operand of a call, on `device`, which has to be the current one: the
    call launches on its current stream."""
    for x, dtype, n, name in checks:
        if x.dtype is not dtype or x.numel() != n or not x.is_contiguous():
            _sized(x, dtype, n, name)
    if device < 0:
        raise ValueError("expected CUDA tensors (this library has no CPU path)")
    for x, _, _, name in checks:
        if x.get_device() != device:
            raise ValueError(f"{name}: on {x.device}, other operands on cuda:{device}")
    if device != _device():
        raise ValueError(f"operands on cuda:{device}, but the current device is cuda:{_device()}")


def _in_32_bits(**sizes: int) -> None:
    """ctypes keeps the low 32 bits of a larger number, which may be a valid other size."""
    for name, n in sizes.items():
        if not -1 << 31 <= n < 1 << 31:
            raise ValueError(f"{name}: {n} is beyond 32 bits")


def pq_block_tables(kv_len, new_len, block_table, free_list, free_head, page: int, tokens: int | None = None,
                    step: PagedStep | None = None) -> PagedStep:
    """Block tables, slot map and positions of one step.  kv_len, new_len i32 [requests]; block_table
    i32 [requests, width], updated in place; free_list i32 [F] page ids, taken from free_head i32 [1] on.
    tokens: rows of the step, at least the sum of new_len; or step: buffers from PagedStep.empty, filled and
    returned."""
    B = kv_len.numel()
    _in_32_bits(page=page)
    if block_table.dim() != 2:
        raise ValueError("block_table: expected a 2-D tensor [requests, width]")
    width, F = block_table.shape[1], free_list.numel()
    checks = ((kv_len, torch.int32, B, "kv_len"), (new_len, torch.int32, B, "new_len"),
              (block_table, torch.int32, B * width, "block_table"), (free_list, torch.int32, F, "free_list"),
              (free_head, torch.int32, 1, "free_head"))
    if step is None:
        if tokens is None or tokens < 0:
            raise ValueError("tokens: expected the rows of the step, or step")
        _operands(kv_len.get_device(), *checks)
        step = PagedStep.empty(B, tokens, kv_len.device)
    else:
        if step.requests != B or (tokens is not None and tokens != step.tokens):
            raise ValueError(f"step: made for {step.requests} requests and {step.tokens} tokens")
        _operands(step.device, *checks)
    q_start, total, slots, pos, head = step._ptrs
    _check("pq_block_tables", lib().pq_block_tables(
        kv_len.data_ptr(), new_len.data_ptr(), B, block_table.data_ptr(), width, free_list.data_ptr(), F,
        free_head.data_ptr(), page, step.tokens, q_start, total, slots, pos, head, _stream()))
    return step


def _token_rows(x: torch.Tensor, heads: int | None, dim: int, what: str) -> tuple[int, int, int]:
    """Rows of f16 head vectors, [T, heads, dim] or [T, heads * dim], dense inside a row; the rows may be slices of
    a wider matrix.  Returns (T, heads, row stride in elements)."""
    if x.dtype != torch.float16:
        raise TypeError(f"{what}: expected torch.float16, got {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) == 3:
        T, H, D = shape
        dense = D == dim and stride[2] == 1 and (H == 1 or stride[1] == dim)
    elif len(shape) == 2:
        T, H, dense = shape[0], shape[1] // dim, shape[1] % dim == 0 and stride[1] == 1
    else:
        dense = False
    if not dense or (heads is not None and H != heads):
        raise ValueError(f"{what}: expected rows of {'heads' if heads is None else heads} x {dim} contiguous values")
    return T, H, (stride[0] if T > 1 else H * dim)


def pq_kv_append(cache: PagedKV, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
    """Writes k, v f16 [T, heads, dim] (or [T, heads * dim]; rows may be slices of a wider matrix) into the cache
    at slots i64 [T]; rows with a negative slot are skipped.  An int8 cache quantizes every head's vector."""
    T, _, ks = _token_rows(k, cache.heads, cache.dim, "k")
    Tv, _, vs = _token_rows(v, cache.heads, cache.dim, "v")
    if Tv != T:
        raise ValueError(f"v: expected {T} rows, got {Tv}")
    _operands(cache.device, (slots, torch.int64, T, "slots"))
    if k.get_device() != cache.device or v.get_device() != cache.device:
        raise ValueError(f"k, v: expected them on the cache's device cuda:{cache.device}")
    _check("pq_kv_append", lib().pq_kv_append(cache._ref, k.data_ptr(), ks, v.data_ptr(), vs, slots.data_ptr(), T,
                                              _stream()))


def pq_kv_read(cache: PagedKV, slots: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """Keys and values at slots i64 [T] as f16 [T, heads, dim]; zeros where a slot is outside the cache."""
    T = slots.numel()
    _operands(cache.device, (slots, torch.int64, T, "slots"))
    k, v = (torch.empty((T, cache.heads, cache.dim), dtype=torch.float16, device=slots.device) for _ in range(2))
    _check("pq_kv_read", lib().pq_kv_read(cache._ref, slots.data_ptr(), T, k.data_ptr(), v.data_ptr(), _stream()))
    return k, v


def pq_attention_workspace_bytes(requests: int, tokens: int, max_q: int, max_kv: int, heads: int, kv_heads: int,
                                 dim: int, sms: int = 148, window: int = 0) -> int:
    """Bytes of workspace with which pq_paged_attention splits the keys as it would with unlimited room, at these
    sizes and this window (another window may want more); 0 if it does not split them.  Host-only, needs no GPU."""
    _in_32_bits(heads=heads, kv_heads=kv_heads, dim=dim, sms=sms, window=window)
    return int(lib().pq_attention_workspace_bytes_window(requests, tokens, max_q, max_kv, heads, kv_heads, dim, sms, window))


def pq_attention_workspace(q: torch.Tensor, cache: PagedKV, requests: int, max_q: int, max_kv: int,
                           window: int = 0) -> torch.Tensor | None:
    """A prepared workspace for pq_paged_attention over these sizes and this window (None where the call has no use
    for one)."""
    T, H, _ = _token_rows(q, None, cache.dim, "q")
    sms = torch.cuda.get_device_properties(q.device).multi_processor_count
    n = pq_attention_workspace_bytes(requests, T, max_q, max_kv, H, cache.heads, cache.dim, sms, window)
    return pq_workspace_init(torch.empty((n,), dtype=torch.uint8, device=q.device)) if n else None


def pq_paged_attention(q: torch.Tensor, cache: PagedKV, block_table: torch.Tensor, q_start: torch.Tensor,
                       kv_len: torch.Tensor, max_q: int, max_kv: int, scale: float | None = None, window: int = 0,
                       out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of a step's tokens over the paged cache that already holds their keys and values.  q f16
    [T, heads, dim] or [T, heads * dim] (rows may be slices of a wider matrix) -> out f16 of the same shape.
    block_table i32 [requests, width], q_start i32 [requests + 1], kv_len i32 [requests] (with the step's own
    tokens); max_q, max_kv: bounds over the requests; scale: 1 / sqrt(dim) by default; window: keys that a row
    sees at most (0: all); workspace: from pq_attention_workspace (without it the keys are not split)."""
    T, H, qs = _token_rows(q, None, cache.dim, "q")
    B = kv_len.numel()
    _in_32_bits(window=window)
    if block_table.dim() != 2:
        raise ValueError("block_table: expected a 2-D tensor [requests, width]")
    width = block_table.shape[1]
    checks = ((block_table, torch.int32, B * width, "block_table"), (q_start, torch.int32, B + 1, "q_start"),
              (kv_len, torch.int32, B, "kv_len"))
    if out is not None:
        checks += ((out, torch.float16, T * H * cache.dim, "out"),)
    ws = ws_bytes = 0
    if workspace is not None:
        ws, ws_bytes = workspace.data_ptr(), workspace.numel()
        checks += ((workspace, torch.uint8, ws_bytes, "workspace"),)
    _operands(cache.device, *checks)
    if q.get_device() != cache.device:
        raise ValueError(f"q: expected it on the cache's device cuda:{cache.device}")
    if out is None:
        out = torch.empty(q.shape, dtype=torch.float16, device=q.device)
    _check("pq_paged_attention", lib().pq_paged_attention(
        q.data_ptr(), qs, H, cache._ref, block_table.data_ptr(), width, q_start.data_ptr(), kv_len.data_ptr(), B, T,
        max_q, max_kv, cache.dim ** -0.5 if scale is None else scale, window, out.data_ptr(), ws, ws_bytes, _stream()))
    return out


# ---- rotary positions and latent attention ---------------------------------------------------------------

LATENT_ROPE = 64   # rotary values of a head of latent attention
NOPE = VALUE = 128   # of the expanded form: the other values of a query or key, values


class _Rotary(ctypes.Structure):   # pq_rotary of include/pq.h
    _fields_ = [("freq", _vp), ("dim", _i32), ("layout", _i32), ("amplitude", ctypes.c_float)]


class _LatentCache(ctypes.Structure):   # pq_latent_cache
    _fields_ = [("data", _vp), ("pages", _i64), ("page", _i32), ("latent", _i32)]


class Rotary:
    """Frequencies of rotary positions over the first `dim` values of a head, made once for a model and kept on `device`.
    layout: "half" turns the values i and i + dim / 2 together, "pairs" 2 i and 2 i + 1.  scaling stretches them by
    `factor` for contexts beyond the `original` length: "none", "linear" (all), "base" (through the base), "bands" (by
    the turns of a pair over the original length, between `low` and `high` in its index) or "waves" (between `low` and `high`
    in original / wavelength).  amplitude multiplies cosines and sines (default: as the scaling has it)."""

    LAYOUTS = {"half": 0, "pairs": 1}
    SCALINGS = {"none": 0, "linear": 1, "base": 2, "bands": 3, "waves": 4}
    __slots__ = ("dim", "layout", "amplitude", "freq", "device", "_struct", "_ref")

    def __init__(self, dim: int, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0,
                 original: float = 0.0, low: float = 1.0, high: float = 32.0, amplitude: float | None = None, device="cuda"):
        _in_32_bits(dim=dim)
        if layout not in self.LAYOUTS:
            raise ValueError(f"layout: expected one of {list(self.LAYOUTS)}, got {layout!r}")
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling: expected one of {list(self.SCALINGS)}, got {scaling!r}")
        host, own = (ctypes.c_int64 * max(dim // 2, 1))(), ctypes.c_float()
        _check("pq_rotary_frequencies", lib().pq_rotary_frequencies(dim, base, self.SCALINGS[scaling], factor, original, low, high,
                                                                    ctypes.addressof(host), ctypes.addressof(own)))
        freq = torch.tensor(list(host), dtype=torch.int64).to(device)
        if not freq.is_cuda:
            raise ValueError("expected CUDA tensors (this library has no CPU path)")
        put = object.__setattr__
        put(self, "dim", dim), put(self, "layout", layout), put(self, "freq", freq), put(self, "device", freq.get_device())
        put(self, "amplitude", own.value if amplitude is None else amplitude)
        put(self, "_struct", _Rotary(freq.data_ptr(), dim, self.LAYOUTS[layout], self.amplitude))
        put(self, "_ref", ctypes.addressof(self._struct))

    def __setattr__(self, name, value):
        raise AttributeError("a Rotary is fixed; make another one")


class LatentKV:
    """A paged cache of latent vectors and turned rotary keys: data f16 [pages, page, latent + 64].  Measures its tensor
    once and keeps it; page a multiple of 16, latent 256 or 512."""

    __slots__ = ("data", "pages", "page", "latent", "device", "_struct", "_ref")

    def __init__(self, data: torch.Tensor):
        if data.dim() != 3:
            raise ValueError("data: expected a 3-D tensor [pages, page, latent + 64]")
        pages, page, wide = data.shape
        _sized(data, torch.float16, data.numel(), "data")
        if wide - LATENT_ROPE not in (256, 512):
            raise ValueError(f"data: expected 256 + {LATENT_ROPE} or 512 + {LATENT_ROPE} values a token, got {wide}")
        _together(data)
        put = object.__setattr__
        put(self, "data", data), put(self, "pages", pages), put(self, "page", page), put(self, "latent", wide - LATENT_ROPE)
        put(self, "device", data.get_device())
        put(self, "_struct", _LatentCache(data.data_ptr(), pages, page, wide - LATENT_ROPE))
        put(self, "_ref", ctypes.addressof(self._struct))

    def __setattr__(self, name, value):
        raise AttributeError("a LatentKV is fixed; make another one over another tensor")

    @classmethod
    def empty(cls, pages: int, page: int, latent: int = 512, device="cuda"):
        """A zero-filled cache."""
        return cls(torch.zeros((pages, page, latent + LATENT_ROPE), dtype=torch.float16, device=device))


def _head_rows(x: torch.Tensor, heads: int | None, dim: int | None, what: str) -> tuple[int, int, int, int, int]:
    """f16 [T, heads, dim], a head's values dense, rows and heads any distance apart.  Returns (T, heads, dim, row stride,
    head stride) in elements."""
    if x.dtype is not torch.float16:
        raise TypeError(f"{what}: expected torch.float16, got {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) != 3 or (stride[2] != 1 and x.numel() > 0) or (heads is not None and shape[1] != heads) or (dim is not None and shape[2] != dim):
        raise ValueError(f"{what}: expected [rows, {'heads' if heads is None else heads}, {'values' if dim is None else dim}] "
                         "with the values of a head contiguous")
    T, H, D = shape
    if (H | D) >> 31:
        _in_32_bits(**{f"{what}'s heads": H, f"{what}'s width": D})
    hs = stride[1] if H > 1 else D
    return T, H, D, (stride[0] if T > 1 else H * hs), hs


def _strided_rows(x: torch.Tensor, width: int, what: str) -> tuple[int, int]:
    """f16 [T, width] or [T, heads, width / heads], dense inside a row.  Returns (T, row stride)."""
    if x.dtype is not torch.float16:
        raise TypeError(f"{what}: expected torch.float16, got {x.dtype}")
    shape, stride = x.shape, x.stride()
    if len(shape) >= 2 and shape[0] == 0:   # whose strides say nothing
        return 0, width
    if len(shape) == 2:
        dense = shape[1] == width and stride[1] == 1
    elif len(shape) == 3:
        dense = shape[1] * shape[2] == width and stride[2] == 1 and (shape[1] == 1 or stride[1] == shape[2])
    else:
        dense = False
    if not dense:
        raise ValueError(f"{what}: expected rows of {width} contiguous values")
    return shape[0], (stride[0] if shape[0] > 1 else width)


def _on(device: int, names: tuple, *tensors) -> None:
    """The tensors whose elements have been measured otherwise lie on `device`, too."""
    for name, x in zip(names, tensors):
        if x is not None and x.get_device() != device:
            raise ValueError(f"{name}: on {x.device}, other operands on cuda:{device}")


def _outputs_for(q: torch.Tensor, out: torch.Tensor | None, T: int, heads: int, dim: int) -> tuple[torch.Tensor, int, int]:
    if out is None:
        return torch.empty((T, heads, dim), dtype=torch.float16, device=q.device), heads * dim, dim
    rows, _, _, os, ohs = _head_rows(out, heads, dim, "out")
    if rows != T:
        raise ValueError(f"out: expected {T} rows, got {rows}")
    return out, os, ohs


def pq_rotate(x: torch.Tensor, pos: torch.Tensor, rotary: Rotary, out: torch.Tensor | None = None) -> torch.Tensor:
    """Rows x f16 [T, heads, width] turned by their positions i32 [T] over the first rotary.dim values of each head -> out
    f16 of the same shape.  Rows and heads may be slices of wider tensors; out may be x itself (in place)."""
    T, H, D, xs, xhs = _head_rows(x, None, None, "x")
    out, os, ohs = _outputs_for(x, out, T, H, D)
    _operands(rotary.device, (pos, torch.int32, T, "pos"))
    _on(rotary.device, ("x", "out"), x, out)
    _check("pq_rotate", lib().pq_rotate(rotary._ref, x.data_ptr(), xs, xhs, H, D, pos.data_ptr(), T, out.data_ptr(), os, ohs, _stream()))
    return out


def _queries(q, out, T: int, dim: int):
    """The optional queries of an append: (out, pointer, strides, heads, pointer, strides)."""
    if q is None:
        if out is not None:
            raise ValueError("out: there are no queries")
        return None, (None, 0, 0, 0, None, 0, 0)
    Tq, H, _, qs, qhs = _head_rows(q, None, dim, "q")
    if Tq != T:
        raise ValueError(f"q: expected {T} rows, got {Tq}")
    out, os, ohs = _outputs_for(q, out, T, H, dim)
    return out, (q.data_ptr(), qs, qhs, H, out.data_ptr(), os, ohs)


def pq_kv_append_rotated(cache: PagedKV, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, pos: torch.Tensor, rotary: Rotary,
                         q: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor | None:
    """pq_kv_append with the keys turned by pos i32 [T] on the way; q f16 [T, heads, dim], where given, is turned beside them
    into out (which may be q) and returned."""
    T, _, ks = _token_rows(k, cache.heads, cache.dim, "k")
    Tv, _, vs = _token_rows(v, cache.heads, cache.dim, "v")
    if Tv != T:
        raise ValueError(f"v: expected {T} rows, got {Tv}")
    out, queries = _queries(q, out, T, cache.dim)
    _operands(cache.device, (slots, torch.int64, T, "slots"), (pos, torch.int32, T, "pos"), (rotary.freq, torch.int64, rotary.dim // 2, "rotary"))
    _on(cache.device, ("k", "v", "q", "out"), k, v, q, out)
    _check("pq_kv_append_rotated", lib().pq_kv_append_rotated(cache._ref, rotary._ref, k.data_ptr(), ks, v.data_ptr(), vs, slots.data_ptr(),
                                                              pos.data_ptr(), T, *queries, _stream()))
    return out


def pq_latent_append(cache: LatentKV, c: torch.Tensor, k_rope: torch.Tensor, slots: torch.Tensor, pos: torch.Tensor, rotary: Rotary,
                     q: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor | None:
    """Writes c f16 [T, latent] and, turned by pos i32 [T], k_rope f16 [T, 64] into the cache at slots i64 [T]; rows with a
    negative slot are skipped.  q f16 [T, heads, 64], where given, is turned beside them into out (which may be q, or
    the end of the latent queries' heads) and returned."""
    T, cs = _strided_rows(c, cache.latent, "c")
    Tk, ks = _strided_rows(k_rope, LATENT_ROPE, "k_rope")
    if Tk != T:
        raise ValueError(f"k_rope: expected {T} rows, got {Tk}")
    out, queries = _queries(q, out, T, LATENT_ROPE)
    _operands(cache.device, (slots, torch.int64, T, "slots"), (pos, torch.int32, T, "pos"), (rotary.freq, torch.int64, rotary.dim // 2, "rotary"))
    _on(cache.device, ("c", "k_rope", "q", "out"), c, k_rope, q, out)
    _check("pq_latent_append", lib().pq_latent_append(cache._ref, rotary._ref, c.data_ptr(), cs, k_rope.data_ptr(), ks, slots.data_ptr(),
                                                      pos.data_ptr(), T, *queries, _stream()))
    return out


def pq_latent_read(cache: LatentKV, slots: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """Latent vectors f16 [T, latent] and turned rotary keys f16 [T, 64] at slots i64 [T]; zeros where a slot is outside the
    cache."""
    T = slots.numel()
    _operands(cache.device, (slots, torch.int64, T, "slots"))
    c, k = (torch.empty((T, n), dtype=torch.float16, device=slots.device) for n in (cache.latent, LATENT_ROPE))
    _check("pq_latent_read", lib().pq_latent_read(cache._ref, slots.data_ptr(), T, c.data_ptr(), k.data_ptr(), _stream()))
    return c, k


def pq_head_linear(x: torch.Tensor, w: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """One matrix per head: x f16 [T, heads, K], w f16 [heads, N, K] -> out f16 [T, heads, N], out[t, h] = w[h] x[t, h].  Rows and
    heads of x and out may be slices of wider tensors."""
    T, H, K, xs, xhs = _head_rows(x, None, None, "x")
    shape = w.shape
    if len(shape) != 3 or shape[0] != H or shape[2] != K:
        raise ValueError(f"w: expected [{H}, N, {K}], got {tuple(shape)}")
    N, device = shape[1], w.get_device()
    out, os, ohs = _outputs_for(x, out, T, H, N)
    _operands(device, (w, torch.float16, H * N * K, "w"))
    _on(device, ("x", "out"), x, out)
    _check("pq_head_linear", lib().pq_head_linear(x.data_ptr(), xs, xhs, w.data_ptr(), H, N, K, T, out.data_ptr(), os, ohs, _stream()))
    return out


def pq_latent_workspace(device="cuda") -> torch.Tensor:
    """A prepared workspace for pq_latent_attention and pq_expanded_attention, of any sizes, on `device`."""
    n = int(lib().pq_latent_workspace_bytes(torch.cuda.get_device_properties(device).multi_processor_count))
    return pq_workspace_init(torch.empty((n,), dtype=torch.uint8, device=device))


def _workspace_check(workspace: torch.Tensor | None):
    """(pointer, bytes, operand checks) of an optional workspace."""
    if workspace is None:
        return None, 0, ()
    return workspace.data_ptr(), workspace.numel(), ((workspace, torch.uint8, workspace.numel(), "workspace"),)


def pq_latent_attention(q: torch.Tensor, cache: LatentKV, block_table: torch.Tensor, q_start: torch.Tensor, kv_len: torch.Tensor,
                        scale: float, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Latent attention, absorbed form, of a step's tokens over the paged latent cache that already holds them.  q f16
    [T, heads, latent + 64], dense, the turned rotary part last -> out f16 [T, heads, latent].  block_table i32
    [requests, width], q_start i32 [requests + 1], kv_len i32 [requests] (with the step's own tokens); workspace: from
    pq_latent_workspace (without it the tokens of a request are not split)."""
    if q.dim() != 3:
        raise ValueError("q: expected a 3-D tensor [rows, heads, latent + 64]")
    T, H, _ = q.shape
    B = kv_len.numel()
    if block_table.dim() != 2:
        raise ValueError("block_table: expected a 2-D tensor [requests, width]")
    width = block_table.shape[1]
    checks = ((q, torch.float16, T * H * (cache.latent + LATENT_ROPE), "q"), (block_table, torch.int32, B * width, "block_table"),
              (q_start, torch.int32, B + 1, "q_start"), (kv_len, torch.int32, B, "kv_len"))
    if out is not None:
        checks += ((out, torch.float16, T * H * cache.latent, "out"),)
    ws, ws_bytes, more = _workspace_check(workspace)
    _operands(cache.device, *checks, *more)
    if out is None:
        out = torch.empty((T, H, cache.latent), dtype=torch.float16, device=q.device)
    _check("pq_latent_attention", lib().pq_latent_attention(q.data_ptr(), H, cache._ref, block_table.data_ptr(), width, q_start.data_ptr(),
                                                            kv_len.data_ptr(), B, T, scale, out.data_ptr(), ws, ws_bytes, _stream()))
    return out


def pq_expanded_attention(q: torch.Tensor, kv: torch.Tensor, k_rope: torch.Tensor, q_start: torch.Tensor, kv_start: torch.Tensor,
                          max_q: int, scale: float, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Latent attention, expanded form: ragged queries q f16 [T, heads, 128 + 64] (the turned rotary part last) over keys and
    values kv f16 [S, heads, 128 + 128] and the turned rotary keys k_rope f16 [S, 64] that all heads share -> out f16
    [T, heads, 128].  Rows of q, kv and k_rope may be slices of wider matrices.  q_start, kv_start i32 [requests + 1]: the
    rows and the keys of each request, whose last row sees all of its keys; max_q: a bound of its rows; workspace: from
    pq_latent_workspace (without it the keys of a request are not split)."""
    if q.dim() != 3:
        raise ValueError(f"q: expected a 3-D tensor [rows, heads, {NOPE + LATENT_ROPE}]")
    H = q.shape[1]
    T, qs = _strided_rows(q, H * (NOPE + LATENT_ROPE), "q")
    S, kvs = _strided_rows(kv, H * (NOPE + VALUE), "kv")
    Sr, krs = _strided_rows(k_rope, LATENT_ROPE, "k_rope")
    if Sr != S:
        raise ValueError(f"k_rope: expected {S} rows, got {Sr}")
    B = q_start.numel() - 1
    checks = ((q_start, torch.int32, B + 1, "q_start"), (kv_start, torch.int32, B + 1, "kv_start"))
    if out is not None:
        checks += ((out, torch.float16, T * H * VALUE, "out"),)
    ws, ws_bytes, more = _workspace_check(workspace)
    _operands(q.get_device(), *checks, *more)
    _on(q.get_device(), ("kv", "k_rope"), kv, k_rope)
    if out is None:
        out = torch.empty((T, H, VALUE), dtype=torch.float16, device=q.device)
    _check("pq_expanded_attention", lib().pq_expanded_attention(q.data_ptr(), qs, H, kv.data_ptr(), kvs, k_rope.data_ptr(), krs, S,
                                                                q_start.data_ptr(), kv_start.data_ptr(), B, T, max_q, scale, out.data_ptr(),
                                                                ws, ws_bytes, _stream()))
    return out


def pq_device_status() -> int:
    """Synchronizes; returns and clears the device status word (0 = ok, 6 = a bounded wait expired)."""
    v = ctypes.c_int(0)
    _check("pq_device_status", lib().pq_device_status(ctypes.byref(v)))
    return int(v.value)
