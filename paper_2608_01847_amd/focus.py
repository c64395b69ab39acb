"""Thin ctypes binding of libfocus (include/focus.h) for torch tensors.

Argument marshalling only: every computation runs in the library's HIP kernels on the caller's
current torch stream. PyTorch provides device memory and streams. Importing this module loads
nothing; the first call opens libfocus.so and raises if it is not built.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

import torch

LIBRARY = Path(__file__).resolve().parent / "libfocus.so"

MXFP4, NVFP4 = 0, 1
F32, BF16 = 0, 1
CALL_SCALES_INIT, CALL_FAKEQUANT_FWD, CALL_FAKEQUANT_BWD = 0, 1, 2
CALL_RECON_GEMM_FWD, CALL_RECON_GEMM_BWD, CALL_EXPORT_PACKED, CALL_ADAMW = 3, 4, 5, 6
CALL_RECON_GEMM_DX, CALL_FAKEQUANT_ACT_BWD, CALL_KL_TOP, CALL_FAKEQUANT_WEIGHTS = 7, 8, 9, 10
CALL_NORM_FWD, CALL_NORM_BWD, CALL_ATTENTION_FWD, CALL_ATTENTION_BWD = 11, 12, 13, 14
CALL_TOKEN_LOGPROBS, CALL_TOKEN_LOGPROBS_BWD, CALL_ATTENTION_FWD_F32, CALL_ATTENTION_BWD_F32 = 15, 16, 17, 18
MAX_WEIGHT_LAYERS = 16
NORM_LAYER, NORM_RMS = 0, 1
MAX_TOP = 64

OK, ERR_NULL, ERR_SHAPE, ERR_DTYPE, ERR_CONFIG, ERR_WORKSPACE, ERR_DOMAIN, ERR_HIP, ERR_SCRATCH = range(9)

EXPORTED = ("focus_workspace_size", "focus_scales_init", "focus_fakequant_fwd", "focus_fakequant_bwd",
            "focus_recon_gemm_fwd", "focus_recon_gemm_fwd_mxfp4", "focus_recon_gemm_fwd_mxfp4_noalloc",
            "focus_recon_gemm_bwd",
            "focus_recon_gemm_bwd_mxfp4", "focus_export_packed", "focus_fakequant_weights", "focus_recon_gemm_dx",
            "focus_fakequant_act_bwd", "focus_kl_top", "focus_adamw_step", "focus_norm_fwd", "focus_norm_bwd",
            "focus_attention_workspace_size", "focus_attention_fwd", "focus_attention_bwd", "focus_token_logprobs",
            "focus_token_logprobs_bwd", "focus_check_flags", "focus_status_string")


class QConfig(ctypes.Structure):
    _fields_ = [("format", ctypes.c_int32), ("sub_block", ctypes.c_int32),
                ("ste_clip", ctypes.c_int32), ("scale_layout", ctypes.c_int32), ("e8m0_rounding", ctypes.c_int32),
                ("code_layout", ctypes.c_int32)]


class WeightLayer(ctypes.Structure):
    _fields_ = [("W", ctypes.c_void_p), ("rows", ctypes.c_int64), ("K", ctypes.c_int64),
                ("s_fp", ctypes.c_void_p), ("c", ctypes.c_void_p), ("alpha", ctypes.c_void_p),
                ("W_hat", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("scale_bytes", ctypes.c_void_p)]


class AdamWConfig(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_float), ("beta1", ctypes.c_float), ("beta2", ctypes.c_float),
                ("eps", ctypes.c_float), ("weight_decay", ctypes.c_float), ("log2_domain", ctypes.c_int32)]


class AttentionConfig(ctypes.Structure):
    _fields_ = [("heads_q", ctypes.c_int32), ("heads_kv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("causal", ctypes.c_int32), ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("dq_stride", ctypes.c_int64), ("dk_stride", ctypes.c_int64), ("dv_stride", ctypes.c_int64)]


class FocusError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_LIB = None


def lib() -> ctypes.CDLL:
    """Opens libfocus.so (built by __graft_entry__.build()); raises if it is missing."""
    global _LIB
    if _LIB is None:
        if not LIBRARY.exists():
            raise RuntimeError(f"{LIBRARY} is not built: run __graft_entry__.build() first")
        L = ctypes.CDLL(str(LIBRARY))
        p, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        q = ctypes.POINTER(QConfig)
        L.focus_workspace_size.argtypes = [i32, q, i64, i64, i64]
        L.focus_workspace_size.restype = sz
        L.focus_scales_init.argtypes = [q, p, i32, i64, i64, p, p, p, p, sz, p]
        L.focus_fakequant_fwd.argtypes = [q, p, i32, i64, i64, p, p, p, p, i32, p, p, p, p, sz, p]
        L.focus_fakequant_bwd.argtypes = [q, p, i64, i64, p, i32, p, p, p, p, p, p, sz, p]
        L.focus_recon_gemm_fwd.argtypes = [p, p, i32, i64, i64, i64, p, p, p, p, p, sz, p]
        L.focus_recon_gemm_fwd_mxfp4.argtypes = [p, p, p, p, i64, i64, i64, p, p, p, p, p, sz, p]
        L.focus_recon_gemm_fwd_mxfp4_noalloc.argtypes = [p, p, p, p, i64, i64, i64, p, p, p, p, p]
        L.focus_recon_gemm_bwd.argtypes = [q, p, p, i32, i64, i64, i64, p, i32, p, p, p, p, p, p, p, sz, p]
        L.focus_recon_gemm_bwd_mxfp4.argtypes = [q, p, p, p, i64, i64, i64, p, i32, p, p, p, p, p, sz, p]
        L.focus_export_packed.argtypes = [q, p, i32, i64, i64, p, p, p, p, p, p, sz, p]
        L.focus_fakequant_weights.argtypes = [q, i32, i32, ctypes.POINTER(WeightLayer), i32, p, sz, p]
        L.focus_recon_gemm_dx.argtypes = [p, p, i32, i64, i64, i64, p, p, sz, p]
        L.focus_fakequant_act_bwd.argtypes = [q, p, i32, i64, i64, p, i32, p, p, sz, p]
        L.focus_kl_top.argtypes = [p, p, i32, i64, i64, i32, p, p, p, sz, p]
        L.focus_adamw_step.argtypes = [ctypes.POINTER(AdamWConfig), i64, i64, p, p, p, p, p, sz, p]
        f32, attn = ctypes.c_float, ctypes.POINTER(AttentionConfig)
        L.focus_norm_fwd.argtypes = [i32, f32, p, p, i32, i64, i64, p, p, i32, p, p, p, p, p, sz, p]
        L.focus_norm_bwd.argtypes = [i32, p, p, i32, i64, i64, p, i32, p, p, p, p, p, p, p, sz, p]
        L.focus_attention_workspace_size.argtypes = [i32, attn, i64, i64, i64]
        L.focus_attention_workspace_size.restype = sz
        L.focus_attention_fwd.argtypes = [attn, p, p, p, i32, i64, i64, p, p, i64, p, p, p, sz, p]
        L.focus_attention_bwd.argtypes = [attn, p, p, p, p, p, p, i32, i64, i64, p, p, i64, p, p, p, p, sz, p]
        L.focus_token_logprobs.argtypes = [p, i32, i64, i64, p, i32, p, p, p, p, p, p, sz, p]
        L.focus_token_logprobs_bwd.argtypes = [p, i32, i64, i64, p, p, p, p, p, p, p, sz, p]
        L.focus_check_flags.argtypes = [p, p]
        L.focus_status_string.argtypes = [i32]
        L.focus_status_string.restype = ctypes.c_char_p
        for name in ("focus_scales_init", "focus_fakequant_fwd", "focus_fakequant_bwd", "focus_recon_gemm_fwd",
                     "focus_recon_gemm_fwd_mxfp4", "focus_recon_gemm_fwd_mxfp4_noalloc", "focus_recon_gemm_bwd",
                     "focus_recon_gemm_bwd_mxfp4",
                     "focus_export_packed", "focus_fakequant_weights", "focus_adamw_step", "focus_check_flags", "focus_recon_gemm_dx", "focus_fakequant_act_bwd",
                     "focus_kl_top", "focus_norm_fwd", "focus_norm_bwd", "focus_attention_fwd", "focus_attention_bwd",
                     "focus_token_logprobs", "focus_token_logprobs_bwd"):
            getattr(L, name).restype = ctypes.c_int
        _LIB = L
    return _LIB


def status_string(status: int) -> str:
    return lib().focus_status_string(status).decode()


SCALES_ROW_MAJOR, SCALES_BLOCK_MAJOR = 0, 1
E8M0_CEIL, E8M0_FLOOR = 0, 1
CODES_ROW_MAJOR, CODES_K_SLAB = 0, 1


def qconfig(fmt: int, sub_block: int, ste_clip: int = 1, scale_layout: int = SCALES_ROW_MAJOR,
            e8m0_rounding: int = 0, code_layout: int = CODES_ROW_MAJOR) -> QConfig:
    return QConfig(fmt, sub_block, ste_clip, scale_layout, e8m0_rounding, code_layout)


def codes_shape(rows: int, K: int, code_layout: int = CODES_ROW_MAJOR) -> tuple:
    """Shape of a packed-code tensor: [rows][K/2], or K-slabs [K/128][rows][64]."""
    return (rows, K // 2) if code_layout == CODES_ROW_MAJOR else (K // 128, rows, 64)


def _slab_dims(codes: torch.Tensor) -> tuple:
    """(rows, K) of codes in K-slabs [K/128][rows][64], the layout of the MXFP4 forward's W operand."""
    if codes.dim() != 3 or codes.shape[2] != 64:
        raise ValueError("the MXFP4 forward takes W codes in K-slabs [K/128][N][64] (code_layout=CODES_K_SLAB)")
    return codes.shape[1], codes.shape[0] * 128


def block_size(fmt: int) -> int:
    return 32 if fmt == MXFP4 else 16


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return BF16
    if t.dtype == torch.float32:
        return F32
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t: torch.Tensor | None):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libfocus must be contiguous")
    return t.data_ptr()


def _stream():
    # the handle of the current device's current stream, without the Stream object around it, whose construction takes
    # 2.8 us of a call's 10
    return ctypes.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))


def _check(status: int, where: str) -> None:
    if status != OK:
        raise FocusError(status, where)


def workspace_size(call: int, q: QConfig, M: int = 0, N: int = 0, K: int = 0) -> int:
    return int(lib().focus_workspace_size(call, ctypes.byref(q), M, N, K))


def workspace(nbytes: int, device="cuda") -> torch.Tensor:
    """A zero-filled workspace (torch's device allocations are at least 256-byte aligned)."""
    ws = torch.zeros(max(nbytes, 256), dtype=torch.uint8, device=device)
    assert ws.data_ptr() % 256 == 0
    return ws


def _ws(ws: torch.Tensor | None, call: int, q: QConfig, M: int, N: int, K: int, device) -> torch.Tensor:
    need = workspace_size(call, q, M, N, K)
    if ws is None or ws.numel() < need:
        ws = workspace(need, device)
    return ws


def scales_init(W: torch.Tensor, fmt: int, sub_block: int, ws=None, out=None, e8m0_rounding: int = 0):
    """Absmax initialisation -> (s_fp [N][K/B], c [N][K/sb] = 1, alpha [1])."""
    N, K = W.shape
    q = qconfig(fmt, sub_block, 1, SCALES_ROW_MAJOR, e8m0_rounding)
    if out is None:
        s_fp = torch.empty(N, K // block_size(fmt), dtype=torch.float32, device=W.device)
        c = torch.empty(N, K // sub_block, dtype=torch.float32, device=W.device)
        alpha = torch.ones(1, dtype=torch.float32, device=W.device)
    else:
        s_fp, c, alpha = out
    ws = _ws(ws, CALL_SCALES_INIT, q, 0, N, K, W.device)
    _check(lib().focus_scales_init(ctypes.byref(q), _ptr(W), _dt(W), N, K, _ptr(s_fp), _ptr(c), _ptr(alpha),
                                   _ptr(ws), ws.numel(), _stream()), "focus_scales_init")
    return s_fp, c, alpha


def fakequant_fwd(X: torch.Tensor, fmt: int, sub_block: int = 8, s_fp=None, c=None, alpha=None,
                  out_dtype=None, want_codes: bool = False, want_scale_bytes: bool = False,
                  want_alpha: bool = False, ste_clip: int = 1, ws=None, out=None, codes_out=None,
                  scales_out=None, scale_layout: int = SCALES_ROW_MAJOR, e8m0_rounding: int = 0,
                  want_x_hat: bool = True, code_layout: int = CODES_ROW_MAJOR):
    """Fake quantisation forward. Weight mode when s_fp is given, dynamic activation mode otherwise.
    codes_out / scales_out: preallocated code and scale-byte outputs (they imply want_codes /
    want_scale_bytes). scale_layout: [rows][K/B] (row-major) or [K/B][rows] (block-major); code_layout:
    [rows][K/2] (row-major) or [K/128][rows][64] (K-slabs). want_x_hat=False (with codes) writes the
    packed form only.

    Returns (x_hat or None, packed_codes or None, scale_bytes or None, alpha_x or None)."""
    rows, K = X.shape
    q = qconfig(fmt, sub_block, ste_clip, scale_layout, e8m0_rounding, code_layout)
    out_dtype = out_dtype or X.dtype
    x_hat = out if out is not None else (torch.empty(rows, K, dtype=out_dtype, device=X.device) if want_x_hat
                                         else None)
    codes = codes_out
    if codes is None and want_codes:
        codes = torch.empty(*codes_shape(rows, K, code_layout), dtype=torch.uint8, device=X.device)
    sbytes = scales_out
    if sbytes is None and want_scale_bytes:
        shape = (rows, K // block_size(fmt)) if scale_layout == SCALES_ROW_MAJOR else (K // block_size(fmt), rows)
        sbytes = torch.empty(*shape, dtype=torch.uint8, device=X.device)
    alpha_out = torch.empty(1, dtype=torch.float32, device=X.device) if want_alpha else None
    ws = _ws(ws, CALL_FAKEQUANT_FWD, q, 0, rows, K, X.device)
    _check(lib().focus_fakequant_fwd(ctypes.byref(q), _ptr(X), _dt(X), rows, K, _ptr(s_fp), _ptr(c), _ptr(alpha),
                                     _ptr(x_hat), _dt(x_hat) if x_hat is not None else _dt(X), _ptr(codes),
                                     _ptr(sbytes), _ptr(alpha_out),
                                     _ptr(ws), ws.numel(), _stream()), "focus_fakequant_fwd")
    return x_hat, codes, sbytes, alpha_out


def fakequant_bwd(G: torch.Tensor, W: torch.Tensor, fmt: int, sub_block: int, s_fp, c=None, alpha=None,
                  ste_clip: int = 1, ws=None, e8m0_rounding: int = 0):
    """Straight-through backward from G = dL/dW_hat (fp32) -> (grad_s, grad_c)."""
    N, K = W.shape
    q = qconfig(fmt, sub_block, ste_clip, SCALES_ROW_MAJOR, e8m0_rounding)
    grad_s = torch.empty(N, K // block_size(fmt), dtype=torch.float32, device=W.device)
    grad_c = torch.empty(N, K // sub_block, dtype=torch.float32, device=W.device)
    ws = _ws(ws, CALL_FAKEQUANT_BWD, q, 0, N, K, W.device)
    _check(lib().focus_fakequant_bwd(ctypes.byref(q), _ptr(G), N, K, _ptr(W), _dt(W), _ptr(s_fp), _ptr(c),
                                     _ptr(alpha), _ptr(grad_s), _ptr(grad_c), _ptr(ws), ws.numel(), _stream()),
           "focus_fakequant_bwd")
    return grad_s, grad_c


def recon_gemm_fwd(X_hat: torch.Tensor, W_hat: torch.Tensor, Y_ref=None, want_col_sq: bool = False, ws=None,
                   out=None, loss=None):
    """Y_hat = X_hat W_hat^T with the MSE epilogue -> (dY (or Y_hat when Y_ref is None), loss, col_sq)."""
    M, K = X_hat.shape
    N = W_hat.shape[0]
    dY = out if out is not None else torch.empty(M, N, dtype=X_hat.dtype, device=X_hat.device)
    loss_t = None
    if Y_ref is not None:
        loss_t = loss if loss is not None else torch.empty(1, dtype=torch.float64, device=X_hat.device)
    col_sq = torch.empty(N, dtype=torch.float64, device=X_hat.device) if want_col_sq else None
    q = qconfig(MXFP4, 8)
    ws = _ws(ws, CALL_RECON_GEMM_FWD, q, M, N, K, X_hat.device)
    _check(lib().focus_recon_gemm_fwd(_ptr(X_hat), _ptr(W_hat), _dt(X_hat), M, N, K, _ptr(Y_ref), _ptr(dY),
                                      _ptr(loss_t), _ptr(col_sq), _ptr(ws), ws.numel(), _stream()),
           "focus_recon_gemm_fwd")
    return dY, loss_t, col_sq


def recon_gemm_fwd_mxfp4(X_codes: torch.Tensor, X_scales: torch.Tensor, W_codes: torch.Tensor, W_scales: torch.Tensor,
                         Y_ref=None, want_col_sq: bool = False, ws=None, out=None, loss=None):
    """The forward from packed MXFP4 operands (X codes [M][K/2], W codes in K-slabs [K/128][N][64],
    block-major E8M0 bytes [K/32][rows]) -> as recon_gemm_fwd."""
    M, K = X_codes.shape[0], X_codes.shape[1] * 2
    N = _slab_dims(W_codes)[0]
    dev = X_codes.device
    dY = out if out is not None else torch.empty(M, N, dtype=torch.bfloat16, device=dev)
    loss_t = None
    if Y_ref is not None:
        loss_t = loss if loss is not None else torch.empty(1, dtype=torch.float64, device=dev)
    col_sq = torch.empty(N, dtype=torch.float64, device=dev) if want_col_sq else None
    ws = _ws(ws, CALL_RECON_GEMM_FWD, qconfig(MXFP4, 8), M, N, K, dev)
    _check(lib().focus_recon_gemm_fwd_mxfp4(_ptr(X_codes), _ptr(X_scales), _ptr(W_codes), _ptr(W_scales), M, N, K,
                                            _ptr(Y_ref), _ptr(dY), _ptr(loss_t), _ptr(col_sq), _ptr(ws), ws.numel(),
                                            _stream()),
           "focus_recon_gemm_fwd_mxfp4")
    return dY, loss_t, col_sq


def recon_gemm_fwd_mxfp4_noalloc(X_codes: torch.Tensor, X_scales: torch.Tensor, W_codes: torch.Tensor,
                                 W_scales: torch.Tensor, Y_ref=None, col_sq=None, out=None, loss=None):
    """recon_gemm_fwd_mxfp4 without a workspace (the library's fixed device scratch instead). The
    library allocates nothing; the caller passes dY (`out`), `loss` when Y_ref is given, and
    optionally `col_sq` [N] float64. -> (dY, loss, col_sq)."""
    M, K = X_codes.shape[0], X_codes.shape[1] * 2
    N = _slab_dims(W_codes)[0]
    if out is None or (Y_ref is not None and loss is None):
        raise ValueError("recon_gemm_fwd_mxfp4_noalloc: pass the outputs (out, and loss with Y_ref)")
    _check(lib().focus_recon_gemm_fwd_mxfp4_noalloc(_ptr(X_codes), _ptr(X_scales), _ptr(W_codes), _ptr(W_scales),
                                                    M, N, K, _ptr(Y_ref), _ptr(out), _ptr(loss), _ptr(col_sq),
                                                    _stream()),
           "focus_recon_gemm_fwd_mxfp4_noalloc")
    return out, loss, col_sq


def recon_gemm_bwd(dY: torch.Tensor, X_hat: torch.Tensor, W: torch.Tensor, fmt: int, sub_block: int, s_fp,
                   c=None, alpha=None, ste_clip: int = 1, want_G: bool = False, ws=None, out=None,
                   e8m0_rounding: int = 0):
    """Fused backward -> (grad_s, grad_c, G or None)."""
    M, K = X_hat.shape
    N = W.shape[0]
    q = qconfig(fmt, sub_block, ste_clip, SCALES_ROW_MAJOR, e8m0_rounding)
    if out is None:
        grad_s = torch.empty(N, K // block_size(fmt), dtype=torch.float32, device=W.device)
        grad_c = torch.empty(N, K // sub_block, dtype=torch.float32, device=W.device)
    else:
        grad_s, grad_c = out
    G = torch.empty(N, K, dtype=torch.float32, device=W.device) if want_G else None
    ws = _ws(ws, CALL_RECON_GEMM_BWD, q, M, N, K, W.device)
    _check(lib().focus_recon_gemm_bwd(ctypes.byref(q), _ptr(dY), _ptr(X_hat), _dt(X_hat), M, N, K, _ptr(W),
                                      _dt(W), _ptr(s_fp), _ptr(c), _ptr(alpha), _ptr(grad_s), _ptr(grad_c),
                                      _ptr(G), _ptr(ws), ws.numel(), _stream()), "focus_recon_gemm_bwd")
    return grad_s, grad_c, G


def recon_gemm_bwd_mxfp4(dY: torch.Tensor, X_codes: torch.Tensor, X_scales: torch.Tensor, W: torch.Tensor,
                         sub_block: int, s_fp, c=None, ste_clip: int = 1, ws=None, out=None, e8m0_rounding: int = 0):
    """Fused backward with X_hat as packed MXFP4 (codes [M][K/2], block-major E8M0 bytes [K/32][M])
    -> (grad_s, grad_c)."""
    M, K = X_codes.shape[0], X_codes.shape[1] * 2
    N = W.shape[0]
    q = qconfig(MXFP4, sub_block, ste_clip, SCALES_ROW_MAJOR, e8m0_rounding)
    if out is None:
        grad_s = torch.empty(N, K // 32, dtype=torch.float32, device=W.device)
        grad_c = torch.empty(N, K // sub_block, dtype=torch.float32, device=W.device)
    else:
        grad_s, grad_c = out
    ws = _ws(ws, CALL_RECON_GEMM_BWD, q, M, N, K, W.device)
    _check(lib().focus_recon_gemm_bwd_mxfp4(ctypes.byref(q), _ptr(dY), _ptr(X_codes), _ptr(X_scales), M, N, K,
                                            _ptr(W), _dt(W), _ptr(s_fp), _ptr(c), _ptr(grad_s), _ptr(grad_c),
                                            _ptr(ws), ws.numel(), _stream()), "focus_recon_gemm_bwd_mxfp4")
    return grad_s, grad_c


def export_packed(W: torch.Tensor, fmt: int, sub_block: int, s_fp, c=None, alpha=None, ws=None, out=None,
                  scale_layout: int = SCALES_ROW_MAJOR, e8m0_rounding: int = 0, code_layout: int = CODES_ROW_MAJOR):
    """Deployable export -> (packed codes [N][K/2] or, in K-slabs, [K/128][N][64]; scale bytes [N][K/B] or,
    block-major, [K/B][N])."""
    N, K = W.shape
    q = qconfig(fmt, sub_block, 1, scale_layout, e8m0_rounding, code_layout)
    if out is None:
        packed = torch.empty(*codes_shape(N, K, code_layout), dtype=torch.uint8, device=W.device)
        shape = (N, K // block_size(fmt)) if scale_layout == SCALES_ROW_MAJOR else (K // block_size(fmt), N)
        sbytes = torch.empty(*shape, dtype=torch.uint8, device=W.device)
    else:
        packed, sbytes = out
    ws = _ws(ws, CALL_EXPORT_PACKED, q, 0, N, K, W.device)
    _check(lib().focus_export_packed(ctypes.byref(q), _ptr(W), _dt(W), N, K, _ptr(s_fp), _ptr(c), _ptr(alpha),
                                     _ptr(packed), _ptr(sbytes), _ptr(ws), ws.numel(), _stream()),
           "focus_export_packed")
    return packed, sbytes


def fakequant_weights(layers, fmt: int, sub_block: int, w_dtype=None, what_dtype=None, ws=None,
                      scale_layout: int = SCALES_ROW_MAJOR, e8m0_rounding: int = 0,
                      code_layout: int = CODES_ROW_MAJOR) -> None:
    """Weight fake quantisation of several layers in one call (focus_fakequant_weights). `layers` is a
    sequence of dicts with keys W, s_fp and optionally c, alpha, W_hat, codes, scale_bytes (device
    tensors; the outputs are written in place). w_dtype / what_dtype default to the first layer's W /
    W_hat dtype."""
    q = qconfig(fmt, sub_block, 1, scale_layout, e8m0_rounding, code_layout)
    arr = (WeightLayer * max(1, len(layers)))()
    for i, l in enumerate(layers):
        W = l["W"]
        arr[i] = WeightLayer(_ptr(W), W.shape[0], W.shape[1], _ptr(l["s_fp"]), _ptr(l.get("c")), _ptr(l.get("alpha")),
                             _ptr(l.get("W_hat")), _ptr(l.get("codes")), _ptr(l.get("scale_bytes")))
    if w_dtype is None:
        w_dtype = _dt(layers[0]["W"]) if layers else BF16
    if what_dtype is None:
        wh = next((l["W_hat"] for l in layers if l.get("W_hat") is not None), None)
        what_dtype = _dt(wh) if wh is not None else w_dtype
    device = layers[0]["W"].device if layers else "cuda"
    ws = _ws(ws, CALL_FAKEQUANT_WEIGHTS, q, 0, 0, 0, device)
    _check(lib().focus_fakequant_weights(ctypes.byref(q), w_dtype, what_dtype, arr, len(layers), _ptr(ws), ws.numel(),
                                         _stream()), "focus_fakequant_weights")


def recon_gemm_dx(dY: torch.Tensor, W_hat: torch.Tensor, ws=None, out=None) -> torch.Tensor:
    """dX_hat = dY W_hat (the input gradient of a linear) -> [M][K] in dY's dtype."""
    M, N = dY.shape
    K = W_hat.shape[1]
    assert W_hat.shape[0] == N and W_hat.dtype == dY.dtype
    dX = out if out is not None else torch.empty(M, K, dtype=dY.dtype, device=dY.device)
    need = workspace_size(CALL_RECON_GEMM_DX, qconfig(MXFP4, 8), M, N, K)
    if ws is None or ws.numel() < need:  # up to 256 MB; only the header's domain flag has to be zero
        ws = torch.empty(need, dtype=torch.uint8, device=dY.device)
        ws[:256].zero_()
    _check(lib().focus_recon_gemm_dx(_ptr(dY), _ptr(W_hat), _dt(dY), M, N, K, _ptr(dX), _ptr(ws), ws.numel(),
                                     _stream()), "focus_recon_gemm_dx")
    return dX


def fakequant_act_bwd(X: torch.Tensor, dX_hat: torch.Tensor, fmt: int, ste_clip: int = 1, e8m0_rounding: int = 0,
                      ws=None, out=None) -> torch.Tensor:
    """Straight-through backward of the activation fake quantisation -> dX (dX_hat's dtype)."""
    rows, K = X.shape
    q = qconfig(fmt, 8, ste_clip, SCALES_ROW_MAJOR, e8m0_rounding)  # the sub-block plays no part here
    dX = out if out is not None else torch.empty_like(dX_hat)
    ws = _ws(ws, CALL_FAKEQUANT_ACT_BWD, q, 0, rows, K, X.device)
    _check(lib().focus_fakequant_act_bwd(ctypes.byref(q), _ptr(X), _dt(X), rows, K, _ptr(dX_hat), _dt(dX_hat),
                                         _ptr(dX), _ptr(ws), ws.numel(), _stream()), "focus_fakequant_act_bwd")
    return dX


def kl_top(Z_student: torch.Tensor, Z_teacher: torch.Tensor, k: int = 1000, ws=None, out=None, loss=None):
    """KL-Top loss of student logits against teacher logits -> (dZ_student, loss [1] fp64)."""
    T, V = Z_student.shape
    assert Z_teacher.shape == Z_student.shape and Z_teacher.dtype == Z_student.dtype
    dZ = out if out is not None else torch.empty_like(Z_student)
    loss_t = loss if loss is not None else torch.empty(1, dtype=torch.float64, device=Z_student.device)
    need = workspace_size(CALL_KL_TOP, qconfig(MXFP4, 8), T, V, 0)
    if ws is None or ws.numel() < need:
        ws = workspace(need, Z_student.device)
    _check(lib().focus_kl_top(_ptr(Z_student), _ptr(Z_teacher), _dt(Z_student), T, V, k, _ptr(dZ), _ptr(loss_t),
                              _ptr(ws), ws.numel(), _stream()), "focus_kl_top")
    return dZ, loss_t


def adamw_step(param: torch.Tensor, grad: torch.Tensor, exp_avg: torch.Tensor, exp_avg_sq: torch.Tensor, t: int,
               lr: float, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.0,
               log2_domain: bool = False, ws=None) -> None:
    """One in-place AdamW step on fp32 `param` (moments in exp_avg / exp_avg_sq, t the 1-based step)."""
    for x in (param, grad, exp_avg, exp_avg_sq):
        assert x.dtype == torch.float32 and x.is_contiguous() and x.numel() == param.numel()
    cfg = AdamWConfig(lr, betas[0], betas[1], eps, weight_decay, int(log2_domain))
    if ws is None:
        ws = workspace(256, param.device)
    _check(lib().focus_adamw_step(ctypes.byref(cfg), t, param.numel(), _ptr(param), _ptr(grad), _ptr(exp_avg),
                                  _ptr(exp_avg_sq), _ptr(ws), ws.numel(), _stream()), "focus_adamw_step")


def norm_workspace_size(T: int, C: int) -> int:
    """Workspace bytes of norm_fwd and norm_bwd on T tokens of C features."""
    return int(lib().focus_workspace_size(CALL_NORM_BWD, None, T, 0, C))


def _sized(ws: torch.Tensor | None, need: int, device) -> torch.Tensor:
    """ws, or where none is given one of `need` bytes of which only the header is cleared. A given workspace is never replaced:
    its header is where the caller looks for the domain flag, and the call refuses one that is too small."""
    if ws is None:
        ws = torch.empty(max(need, 256), dtype=torch.uint8, device=device)  # need is 0 for arguments that the call refuses
        ws[:256].zero_()
    return ws


def _one_gpu(where: str, first: torch.Tensor, *rest) -> None:
    """All tensors (None: not given) lie on one GPU, the current one: a host address would reach a kernel otherwise, or a
    kernel run on another GPU's stream, in no order with the work on the tensors."""
    d = first.get_device()
    if d < 0 or any(t is not None and t.get_device() != d for t in rest):
        raise ValueError(f"{where}: tensors of one GPU expected")
    if d != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors of GPU {d} while GPU {torch.cuda.current_device()} is the current one")


def norm_fwd(X: torch.Tensor, weight: torch.Tensor, bias=None, residual=None, kind: int = NORM_LAYER, eps: float = 1e-5,
             want_stats: bool = True, ws=None, out=None, h_out=None):
    """Layer norm (NORM_LAYER) or RMS norm (NORM_RMS) over the last dimension of X [T][C], with an optional residual sum
    H = X + residual in front of it -> (Y, H or None, mean [T] or None, rstd [T] or None). `out` / `h_out`: preallocated
    Y / H. The statistics are fp32 (mean: layer norm only; neither without want_stats)."""
    T, C = X.shape
    for t in (residual, out, h_out):
        if t is not None and (t.shape != X.shape or t.dtype != X.dtype):
            raise ValueError("norm_fwd: residual, out and h_out have X's shape and dtype")
    if weight.shape != (C,) or (bias is not None and (bias.shape != (C,) or bias.dtype != weight.dtype)):
        raise ValueError("norm_fwd: weight and bias are [C] of one dtype")
    if h_out is not None and residual is None:
        raise ValueError("norm_fwd: h_out without a residual")
    _one_gpu("norm_fwd", X, weight, bias, residual, ws, out, h_out)
    Y = out if out is not None else torch.empty_like(X)
    H = (h_out if h_out is not None else torch.empty_like(X)) if residual is not None else None
    mean = rstd = None
    if want_stats:
        rstd = torch.empty(T, dtype=torch.float32, device=X.device)
        mean = torch.empty(T, dtype=torch.float32, device=X.device) if kind == NORM_LAYER else None
    ws = _sized(ws, 256, X.device)
    _check(lib().focus_norm_fwd(kind, eps, _ptr(X), _ptr(residual), _dt(X), T, C, _ptr(weight), _ptr(bias), _dt(weight),
                                _ptr(H), _ptr(Y), _ptr(mean), _ptr(rstd), _ptr(ws), ws.numel(), _stream()),
           "focus_norm_fwd")
    return Y, H, mean, rstd


def norm_bwd(dY: torch.Tensor, H: torch.Tensor, weight: torch.Tensor, mean, rstd: torch.Tensor, d_residual=None,
             kind: int = NORM_LAYER, want_bias: bool = False, ws=None, out=None, dw_out=None, db_out=None):
    """Backward of norm_fwd on its input H (the residual sum, or X where there was none) -> (dX, dweight [C] fp32,
    dbias [C] fp32 or None). d_residual: the gradient that reaches H past the norm; dX is the gradient of X and of the
    residual alike. dX may be dY's or d_residual's own tensor (`out`)."""
    T, C = H.shape
    for t in (dY, d_residual, out):
        if t is not None and (t.shape != H.shape or t.dtype != H.dtype):
            raise ValueError("norm_bwd: dY, d_residual and out have H's shape and dtype")
    for t, n in ((weight, C), (mean, T), (rstd, T), (dw_out, C), (db_out, C)):
        if t is not None and t.shape != (n,):
            raise ValueError("norm_bwd: weight and its gradients are [C], mean and rstd [T]")
    for t in (mean, rstd, dw_out, db_out):
        if t is not None and t.dtype != torch.float32:
            raise TypeError("norm_bwd: statistics and parameter gradients are float32")
    _one_gpu("norm_bwd", H, dY, weight, mean, rstd, d_residual, ws, out, dw_out, db_out)
    dX = out if out is not None else torch.empty_like(H)
    dw = dw_out if dw_out is not None else torch.empty(C, dtype=torch.float32, device=H.device)
    db = db_out
    if db is None and want_bias:
        db = torch.empty(C, dtype=torch.float32, device=H.device)
    ws = _sized(ws, norm_workspace_size(T, C), H.device)
    _check(lib().focus_norm_bwd(kind, _ptr(dY), _ptr(H), _dt(H), T, C, _ptr(weight), _dt(weight), _ptr(mean), _ptr(rstd),
                                _ptr(d_residual), _ptr(dX), _ptr(dw), _ptr(db), _ptr(ws), ws.numel(), _stream()),
           "focus_norm_bwd")
    return dX, dw, db


def _heads(t: torch.Tensor, name: str) -> tuple:
    """(pointer, elements between tokens) of [tokens][heads][head_dim] whose tokens may lie apart (a slice of a fused
    product); a token's heads are contiguous."""
    if t.dim() != 3:
        raise ValueError(f"{name}: [tokens][heads][head_dim] expected")
    n, h, d = t.shape
    if n and ((d > 1 and t.stride(2) != 1) or (h > 1 and t.stride(1) != d)):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    stride = t.stride(0) if n > 1 else h * d
    if stride < h * d:
        raise ValueError(f"{name}: tokens overlap")
    return t.data_ptr(), stride


def _attention_config(q, k, causal, scale, strides=(0,) * 6) -> AttentionConfig:
    d = q.shape[2]
    return AttentionConfig(q.shape[1], k.shape[1], d, int(causal), d ** -0.5 if scale is None else scale, 0, *strides)


def _ends(cu: torch.Tensor | None, name: str):
    if cu is None:
        return None, 1
    if cu.dtype != torch.int32 or cu.dim() != 1 or cu.numel() < 1:
        raise ValueError(f"{name}: a tensor of n_seq + 1 int32 ends expected")
    return _ptr(cu), cu.numel() - 1


def _attention_inputs(q, k, v, cu_q, cu_k):
    if k.shape != v.shape or q.shape[2] != k.shape[2] or not (q.dtype == k.dtype == v.dtype):
        raise ValueError("attention: q [Tq][Hq][D], k and v [Tk][Hkv][D] of one dtype expected")
    if cu_k is None:
        cu_k = cu_q
    pq, n = _ends(cu_q, "cu_q")
    pk, nk = _ends(cu_k, "cu_k")
    if n != nk or (cu_q is None) != (cu_k is None):
        raise ValueError("attention: cu_q and cu_k name the same sequences")
    return pq, pk, n


def attention_workspace_size(q: torch.Tensor, k: torch.Tensor, n_seq: int = 1) -> int:
    """Workspace bytes of attention_fwd and attention_bwd on tensors of these shapes and dtype, packed into n_seq sequences. Fewer
    bf16 queries may need more (their keys are split): take the largest over the shapes that are called."""
    c = _attention_config(q, k, 0, 1.0)
    return max(_attention_ws_bytes(call, c, q, k, n_seq) for call in (CALL_ATTENTION_FWD, CALL_ATTENTION_BWD))


def _attention_ws_bytes(call: int, cfg: AttentionConfig, q: torch.Tensor, k: torch.Tensor, n_seq: int) -> int:
    if _dt(q) == F32:
        call = {CALL_ATTENTION_FWD: CALL_ATTENTION_FWD_F32, CALL_ATTENTION_BWD: CALL_ATTENTION_BWD_F32}[call]
    return int(lib().focus_attention_workspace_size(call, ctypes.byref(cfg), q.shape[0], k.shape[0], n_seq))


def attention_fwd(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, cu_q=None, cu_k=None, causal: bool = True,
                  scale: float | None = None, want_lse: bool = True, ws=None, out=None, lse=None):
    """Attention of q [Tq][Hq][D] over k, v [Tk][Hkv][D], sequences packed one after the other with ends cu_q, cu_k
    (int32 [n_seq + 1] on the device; cu_k defaults to cu_q, both None: one sequence) -> (O [Tq][Hq][D], lse [Hq][Tq]
    fp32 or None). q, k and v may be slices of one fused product (tokens apart); `out` may be q. scale defaults to D ** -0.5."""
    pq, pk, n = _attention_inputs(q, k, v, cu_q, cu_k)
    (aq, sq), (ak, sk), (av, sv) = _heads(q, "q"), _heads(k, "k"), _heads(v, "v")
    cfg = _attention_config(q, k, causal, scale, (sq, sk, sv, 0, 0, 0))
    O = out if out is not None else torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if O.shape != q.shape or O.dtype != q.dtype:
        raise ValueError("attention_fwd: out has q's shape and dtype")
    if lse is None and want_lse:
        lse = torch.empty(q.shape[1], q.shape[0], dtype=torch.float32, device=q.device)
    if lse is not None and (lse.shape != (q.shape[1], q.shape[0]) or lse.dtype != torch.float32):
        raise ValueError("attention_fwd: lse is float32 [Hq][Tq]")
    _one_gpu("attention_fwd", q, k, v, cu_q, cu_k, ws, out, lse)
    ws = _sized(ws, _attention_ws_bytes(CALL_ATTENTION_FWD, cfg, q, k, n), q.device)
    _check(lib().focus_attention_fwd(ctypes.byref(cfg), aq, ak, av, _dt(q), q.shape[0], k.shape[0], pq, pk, n, _ptr(O),
                                     _ptr(lse), _ptr(ws), ws.numel(), _stream()), "focus_attention_fwd")
    return O, lse


def attention_bwd(dO: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, O: torch.Tensor, lse: torch.Tensor,
                  cu_q=None, cu_k=None, causal: bool = True, scale: float | None = None, ws=None, out=None):
    """Backward of attention_fwd from its outputs O and lse -> (dq, dk, dv) in q's dtype. `out`: preallocated (dq, dk, dv),
    which may be slices of one fused gradient and share no memory with each other or with an input."""
    pq, pk, n = _attention_inputs(q, k, v, cu_q, cu_k)
    if dO.shape != q.shape or O.shape != q.shape or lse.shape != (q.shape[1], q.shape[0]):
        raise ValueError("attention_bwd: dO and O have q's shape, lse is [Hq][Tq]")
    if dO.dtype != q.dtype or O.dtype != q.dtype or lse.dtype != torch.float32:
        raise TypeError("attention_bwd: dO and O have q's dtype, lse is float32")
    if out is None:
        out = tuple(torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    dq, dk, dv = out
    for g, t in ((dq, q), (dk, k), (dv, v)):
        if g.shape != t.shape or g.dtype != t.dtype:
            raise ValueError("attention_bwd: the gradients have the shapes and dtype of q, k, v")
    _one_gpu("attention_bwd", q, k, v, dO, O, lse, cu_q, cu_k, ws, dq, dk, dv)
    ptrs = [_heads(t, name) for t, name in ((q, "q"), (k, "k"), (v, "v"), (dq, "dq"), (dk, "dk"), (dv, "dv"))]
    cfg = _attention_config(q, k, causal, scale, tuple(s for _, s in ptrs))
    ws = _sized(ws, _attention_ws_bytes(CALL_ATTENTION_BWD, cfg, q, k, n), q.device)
    (aq, ak, av, adq, adk, adv) = (a for a, _ in ptrs)
    _check(lib().focus_attention_bwd(ctypes.byref(cfg), _ptr(dO), aq, ak, av, _ptr(O), _ptr(lse), _dt(q), q.shape[0],
                                     k.shape[0], pq, pk, n, adq, adk, adv, _ptr(ws), ws.numel(), _stream()),
           "focus_attention_bwd")
    return dq, dk, dv


def token_logprobs_workspace_size(T: int, V: int, top: int = 0) -> int:
    """Workspace bytes of token_logprobs (and token_logprobs_bwd) on T rows of V logits."""
    return int(lib().focus_workspace_size(CALL_TOKEN_LOGPROBS, None, T, V, top))


def _targets(target, T: int):
    if target is not None and (target.shape != (T,) or target.dtype != torch.int64):
        raise ValueError("targets are int64 [T]")
    return _ptr(target)


def token_logprobs(Z: torch.Tensor, target=None, top: int = 0, ws=None):
    """Log probabilities under logits Z [T][V] -> (logp [T] of the tokens `target` (int64; below zero: left out, 0) or
    None, entropy [T], lse [T], top_logp [T][top] or None, top_index [T][top] int32 or None), fp32."""
    T, V = Z.shape
    f32 = dict(dtype=torch.float32, device=Z.device)
    pt = _targets(target, T)
    _one_gpu("token_logprobs", Z, target, ws)
    logp = torch.empty(T, **f32) if target is not None else None
    entropy, lse = torch.empty(T, **f32), torch.empty(T, **f32)
    top_logp = top_index = None
    if top:
        top_logp = torch.empty(T, max(0, top), **f32)
        top_index = torch.empty(T, max(0, top), dtype=torch.int32, device=Z.device)
    ws = _sized(ws, token_logprobs_workspace_size(T, V, top), Z.device)
    _check(lib().focus_token_logprobs(_ptr(Z), _dt(Z), T, V, pt, top, _ptr(logp), _ptr(entropy), _ptr(lse), _ptr(top_logp),
                                      _ptr(top_index), _ptr(ws), ws.numel(), _stream()), "focus_token_logprobs")
    return logp, entropy, lse, top_logp, top_index


def token_logprobs_bwd(Z: torch.Tensor, target, lse: torch.Tensor, entropy=None, d_logp=None, d_entropy=None, ws=None,
                       out=None) -> torch.Tensor:
    """Gradient of token_logprobs' logp and entropy -> dZ [T][V] in Z's dtype (`out` may be Z itself)."""
    T, V = Z.shape
    for t in (lse, entropy, d_logp, d_entropy):
        if t is not None and (t.shape != (T,) or t.dtype != torch.float32):
            raise ValueError("token_logprobs_bwd: lse, entropy and their gradients are float32 [T]")
    dZ = out if out is not None else torch.empty_like(Z)
    if dZ.shape != Z.shape or dZ.dtype != Z.dtype:
        raise ValueError("token_logprobs_bwd: out has Z's shape and dtype")
    _one_gpu("token_logprobs_bwd", Z, target, lse, entropy, d_logp, d_entropy, ws, out)
    ws = _sized(ws, 256, Z.device)
    _check(lib().focus_token_logprobs_bwd(_ptr(Z), _dt(Z), T, V, _targets(target, T), _ptr(lse), _ptr(entropy), _ptr(d_logp),
                                          _ptr(d_entropy), _ptr(dZ), _ptr(ws), ws.numel(), _stream()),
           "focus_token_logprobs_bwd")
    return dZ


def check_flags(ws: torch.Tensor) -> int:
    """Synchronises the current stream; returns OK or ERR_DOMAIN (and clears the flag)."""
    return int(lib().focus_check_flags(_ptr(ws), _stream()))
