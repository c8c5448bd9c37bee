"""ctypes binding of libreqat (C ABI in include/reqat.h).

Two layers:
  * ``reqat_quantize_fp4``, ``reqat_fakequant_fp4``, ``reqat_gemm_w4a4``, ... --
    the C entry points under the same names, taking raw device pointers
    (ints) and sizes; they return the C status code.
  * ``quantize``, ``fakequant``, ``gemm`` -- torch-tensor conveniences that
    allocate outputs with torch, pass ``data_ptr()`` and the current HIP
    stream, and raise ``ReqatError`` on a non-OK status.

Every step of the computation runs in the HIP library; this module only
marshals arguments.  It raises at load time when the library is missing.
"""
from __future__ import annotations

import array
import ctypes
import functools
import operator
import os

import torch

NVFP4 = 0
MXFP4 = 1
BLOCK = {NVFP4: 16, MXFP4: 32}
DT_F32 = 0
DT_BF16 = 1
TS_COMPUTE = 0
TS_GIVEN = 1

STATUS = {0: "REQAT_OK", 1: "REQAT_E_NULL", 2: "REQAT_E_SHAPE", 3: "REQAT_E_ALIGN",
          4: "REQAT_E_ENUM", 5: "REQAT_E_UNSUPPORTED", 6: "REQAT_E_HIP", 7: "REQAT_E_TOO_LARGE"}
NOALLOC_SCRATCH_BYTES = 8 << 20          # REQAT_NOALLOC_SCRATCH_BYTES

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libreqat.so")

# every symbol include/reqat.h declares, with its ctypes signature
_VP = ctypes.c_void_p
_I64 = ctypes.c_int64
_INT = ctypes.c_int
_F32 = ctypes.c_float
SIGNATURES = {
    "reqat_quantize_fp4": (_INT, [_INT, _VP, _I64, _I64, _I64, _VP, _VP, _VP, _INT, _VP, _VP]),
    "reqat_fakequant_fp4": (_INT, [_INT, _VP, _I64, _I64, _I64, _VP, _I64, _VP, _INT, _VP, _VP]),
    "reqat_quantize_fakequant_fp4": (_INT, [_INT, _VP, _I64, _I64, _I64, _VP, _VP, _VP, _I64, _VP, _INT, _VP,
                                            _VP]),
    "reqat_gemm_w4a4": (_INT, [_INT, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _INT,
                               _I64, _VP]),
    "reqat_linear_w4a4": (_INT, [_INT, _I64, _I64, _I64, _VP, _I64, _VP, _INT, _VP, _VP, _VP, _VP,
                                 _INT, _I64, _VP, _VP]),
    "reqat_linear_workspace_bytes": (ctypes.c_size_t, [_INT, _I64, _I64]),
    "reqat_w4a4_packed_bytes": (ctypes.c_size_t, [_INT, _I64, _I64]),
    "reqat_pack_w4a4": (_INT, [_INT, _VP, _VP, _I64, _I64, _VP, _VP]),
    "reqat_gemm_w4a4_packed": (_INT, [_INT, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP, _VP, _INT, _I64, _VP]),
    "reqat_linear_w4a4_packed": (_INT, [_INT, _I64, _I64, _I64, _VP, _I64, _VP, _INT, _VP, _VP, _VP, _INT, _I64,
                                        _VP, _VP]),
    "reqat_linear_w4a4_noalloc": (_INT, [_INT, _I64, _I64, _I64, _VP, _I64, _VP, _INT, _VP, _VP, _VP, _VP,
                                         _INT, _I64, _VP]),
    "reqat_sem_loss": (_INT, [_VP, _I64, _I64, _I64, _VP, ctypes.c_float, ctypes.c_float, _VP, _VP, _VP, _VP]),
    "reqat_sem_loss_backward": (_INT, [_VP, _I64, _I64, _I64, _VP, _VP, _VP, ctypes.c_float, ctypes.c_float,
                                       _VP, _INT, _I64, _VP]),
    "reqat_quantize_kv4": (_INT, [_VP, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _INT, _VP, _VP]),
    "reqat_fakequant_kv4": (_INT, [_VP, _I64, _I64, _I64, _VP, _VP, _I64, _VP, _INT, _VP, _VP]),
    "reqat_kv4_append": (_INT, [_VP, _I64, _VP, _VP, _I64, _VP, _I64, _VP, _I64, _I64, _VP, _I64, _VP, _VP, _VP, _I64,
                                _VP]),
    "reqat_kv4_gather": (_INT, [_VP, _I64, _VP, _VP, _I64, _VP, _I64, _INT, _VP]),
    "reqat_kv4_attention": (_INT, [_VP, _I64, _I64, _VP, _I64, _I64, _VP, _VP, _VP, _I64, _I64, _I64, _I64, _INT,
                                   ctypes.c_float, _VP, _I64, _VP, _VP, _VP]),
    "reqat_kv4_attention_workspace_bytes": (ctypes.c_size_t, [_I64, _I64, _I64, _I64, _I64, _I64, _I64]),
    "reqat_gemm_w4a16": (_INT, [_I64, _I64, _I64, _VP, _I64, _VP, _VP, _VP, _INT, _I64, _VP, _VP]),
    "reqat_w4a16_workspace_bytes": (ctypes.c_size_t, [_I64, _I64, _I64]),
    "reqat_w4a16_packed_bytes": (ctypes.c_size_t, [_I64, _I64]),
    "reqat_pack_w4a16": (_INT, [_VP, _VP, _I64, _I64, _VP, _VP]),
    "reqat_gemm_w4a16_packed": (_INT, [_I64, _I64, _I64, _VP, _I64, _VP, _VP, _INT, _I64, _VP, _VP]),
    "reqat_quantize_mxfp4_rht": (_INT, [_VP, _I64, _I64, _I64, ctypes.c_uint32, _VP, _VP, _VP]),
    "reqat_fakequant_mxfp4_rht": (_INT, [_VP, _I64, _I64, _I64, ctypes.c_uint32, _VP, _I64, _VP]),
    "reqat_policy_loss": (_INT, [_VP, _INT, _I64, _I64, _I64, _VP, _VP, _VP, _VP, _VP, _F32, _F32, _F32, _F32, _VP, _VP, _VP,
                                 _I64, _VP, _VP]),
    "reqat_policy_loss_workspace_bytes": (ctypes.c_size_t, [_INT, _I64, _I64]),
    "reqat_policy_loss_backward": (_INT, [_VP, _INT, _I64, _I64, _I64, _VP, _VP, _F32, _VP, _VP, _I64, _VP]),
    "reqat_layer_norm": (_INT, [_VP, _INT, _I64, _I64, _I64, _VP, _VP, _INT, _F32, _INT, _VP, _I64, _VP, _VP]),
    "reqat_layer_norm_workspace_bytes": (ctypes.c_size_t, [_INT, _I64, _I64, _INT]),
    "reqat_layer_norm_backward": (_INT, [_VP, _I64, _VP, _I64, _INT, _I64, _I64, _VP, _INT, _VP, _INT, _VP, _I64, _VP, _VP,
                                         _VP, _VP]),
    "reqat_embedding": (_INT, [_VP, _I64, _VP, _INT, _I64, _I64, _I64, _F32, _VP, _I64, _VP]),
    "reqat_embedding_workspace_bytes": (ctypes.c_size_t, [_I64, _I64, _I64]),
    "reqat_embedding_backward": (_INT, [_VP, _INT, _I64, _VP, _I64, _I64, _I64, _F32, _VP, _INT, _I64, _INT, _VP, _VP]),
    "reqat_adamw_step": (_INT, [_VP, _I64, _INT, _INT, _INT, _VP, _VP, _VP, _VP]),
    "reqat_adamw_coefficients": (_INT, [_VP, _VP, _VP, _VP, _VP]),
    "reqat_adamw_moments": (_INT, [_VP, _VP, _VP, _VP, _I64, _VP, _VP, _VP]),
    "reqat_workspace_bytes": (ctypes.c_size_t, []),
    "reqat_status_str": (ctypes.c_char_p, [_INT]),
    "reqat_abi_version": (_INT, []),
}

_lib = None


class ReqatError(RuntimeError):
    def __init__(self, status: int, where: str):
        super().__init__("%s failed: %s" % (where, STATUS.get(status, status)))
        self.status = status


def load(path: str = LIB_PATH):
    """Load libreqat.so once; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError("libreqat.so is not built (%s); run python -m paper_2606_15682_amd.build"
                           % path)
    lib = ctypes.CDLL(path)
    for name, (res, args) in SIGNATURES.items():
        f = getattr(lib, name)
        f.restype = res
        f.argtypes = args
    _lib = lib
    return lib


# ------------------------------------------------------------------ raw C entry points

def reqat_quantize_fp4(fmt, x, rows, cols, ldx, codes, scales, tensor_scale, ts, workspace, stream):
    return load().reqat_quantize_fp4(fmt, x, rows, cols, ldx, codes, scales, tensor_scale, ts,
                                     workspace, stream)


def reqat_fakequant_fp4(fmt, x, rows, cols, ldx, y, ldy, tensor_scale, ts, workspace, stream):
    return load().reqat_fakequant_fp4(fmt, x, rows, cols, ldx, y, ldy, tensor_scale, ts, workspace,
                                      stream)


def reqat_quantize_fakequant_fp4(fmt, x, rows, cols, ldx, codes, scales, y, ldy, tensor_scale, ts, workspace,
                                 stream):
    return load().reqat_quantize_fakequant_fp4(fmt, x, rows, cols, ldx, codes, scales, y, ldy, tensor_scale, ts,
                                               workspace, stream)


def reqat_gemm_w4a4(fmt, M, N, K, a_codes, a_scales, a_ts, b_codes, b_scales, b_ts, y, y_dtype,
                    ldy, stream):
    return load().reqat_gemm_w4a4(fmt, M, N, K, a_codes, a_scales, a_ts, b_codes, b_scales, b_ts, y,
                                  y_dtype, ldy, stream)


def reqat_linear_w4a4(fmt, M, N, K, x, ldx, x_ts, ts, w_codes, w_scales, w_ts, y, y_dtype, ldy,
                      workspace, stream):
    return load().reqat_linear_w4a4(fmt, M, N, K, x, ldx, x_ts, ts, w_codes, w_scales, w_ts, y,
                                    y_dtype, ldy, workspace, stream)


def reqat_sem_loss(logits, T, V, ld, targets, lam, eps, stats, weights, loss, stream):
    return load().reqat_sem_loss(logits, T, V, ld, targets, lam, eps, stats, weights, loss, stream)


def reqat_sem_loss_backward(logits, T, V, ld, targets, stats, weights, lam, scale, grad, grad_dtype, ldg, stream):
    return load().reqat_sem_loss_backward(logits, T, V, ld, targets, stats, weights, lam, scale, grad, grad_dtype,
                                          ldg, stream)


def reqat_quantize_kv4(x, rows, cols, ldx, shift, codes, scales, tensor_scale, ts, workspace, stream):
    return load().reqat_quantize_kv4(x, rows, cols, ldx, shift, codes, scales, tensor_scale, ts, workspace,
                                     stream)


def reqat_fakequant_kv4(x, rows, cols, ldx, shift, y, ldy, tensor_scale, ts, workspace, stream):
    return load().reqat_fakequant_kv4(x, rows, cols, ldx, shift, y, ldy, tensor_scale, ts, workspace, stream)


class Kv4CacheStruct(ctypes.Structure):
    """reqat_kv4_cache of the C ABI; the calls below take it by reference."""
    _fields_ = [("k_codes", _VP), ("k_scales", _VP), ("v_codes", _VP), ("v_scales", _VP),
                ("k_tensor_scale", _VP), ("v_tensor_scale", _VP), ("k_shift", _VP),
                ("num_pages", _I64), ("page_size", _I64), ("kv_heads", _I64), ("head_dim", _I64)]


def _cache_ref(cache):
    return None if cache is None else ctypes.addressof(cache)


def reqat_kv4_append(cache, T, slots, k, ldk, v, ldv, q, ldq, q_heads, q_out, ldq_out, rope_cos, rope_sin, positions,
                     rope_len, stream):
    return load().reqat_kv4_append(_cache_ref(cache), T, slots, k, ldk, v, ldv, q, ldq, q_heads, q_out, ldq_out,
                                   rope_cos, rope_sin, positions, rope_len, stream)


def reqat_kv4_gather(cache, T, slots, k_out, ldk, v_out, ldv, add_shift, stream):
    return load().reqat_kv4_gather(_cache_ref(cache), T, slots, k_out, ldk, v_out, ldv, add_shift, stream)


def reqat_kv4_attention(cache, B, T, q, ldq, q_heads, q_start, kv_len, block_table, ld_table, table_cols, max_q,
                        max_kv, causal, sm_scale, out, ldo, lse, workspace, stream):
    return load().reqat_kv4_attention(_cache_ref(cache), B, T, q, ldq, q_heads, q_start, kv_len, block_table, ld_table,
                                      table_cols, max_q, max_kv, causal, sm_scale, out, ldo, lse, workspace, stream)


def reqat_kv4_attention_workspace_bytes(B, T, max_q, max_kv, q_heads, kv_heads, head_dim) -> int:
    return load().reqat_kv4_attention_workspace_bytes(B, T, max_q, max_kv, q_heads, kv_heads, head_dim)


def reqat_gemm_w4a16(M, N, K, x, ldx, w_codes, w_scales, y, y_dtype, ldy, workspace, stream):
    return load().reqat_gemm_w4a16(M, N, K, x, ldx, w_codes, w_scales, y, y_dtype, ldy, workspace, stream)


def reqat_w4a16_workspace_bytes(M, N, K) -> int:
    return load().reqat_w4a16_workspace_bytes(M, N, K)


def reqat_w4a16_packed_bytes(N, K) -> int:
    return load().reqat_w4a16_packed_bytes(N, K)


def reqat_pack_w4a16(w_codes, w_scales, N, K, packed, stream):
    return load().reqat_pack_w4a16(w_codes, w_scales, N, K, packed, stream)


def reqat_gemm_w4a16_packed(M, N, K, x, ldx, packed, y, y_dtype, ldy, workspace, stream):
    return load().reqat_gemm_w4a16_packed(M, N, K, x, ldx, packed, y, y_dtype, ldy, workspace, stream)


def reqat_quantize_mxfp4_rht(x, rows, cols, ldx, signs, codes, scales, stream):
    return load().reqat_quantize_mxfp4_rht(x, rows, cols, ldx, signs, codes, scales, stream)


def reqat_fakequant_mxfp4_rht(x, rows, cols, ldx, signs, y, ldy, stream):
    return load().reqat_fakequant_mxfp4_rht(x, rows, cols, ldx, signs, y, ldy, stream)


def reqat_policy_loss(logits, dtype, T, V, ld, targets, old_logp, advantages, ref_logp, weights, clip_low, clip_high,
                      kl_coef, temperature, stats, loss, grad, ldg, workspace, stream):
    return load().reqat_policy_loss(logits, dtype, T, V, ld, targets, old_logp, advantages, ref_logp, weights, clip_low,
                                    clip_high, kl_coef, temperature, stats, loss, grad, ldg, workspace, stream)


def reqat_policy_loss_workspace_bytes(dtype, T, V) -> int:
    return load().reqat_policy_loss_workspace_bytes(dtype, T, V)


def reqat_policy_loss_backward(logits, dtype, T, V, ld, targets, stats, temperature, grad_loss, grad, ldg, stream):
    return load().reqat_policy_loss_backward(logits, dtype, T, V, ld, targets, stats, temperature, grad_loss, grad, ldg,
                                             stream)


def reqat_layer_norm(x, dtype, rows, cols, ldx, weight, bias, w_dtype, eps, center, y, ldy, stats, stream):
    return load().reqat_layer_norm(x, dtype, rows, cols, ldx, weight, bias, w_dtype, eps, center, y, ldy, stats, stream)


def reqat_layer_norm_workspace_bytes(dtype, rows, cols, bias) -> int:
    return load().reqat_layer_norm_workspace_bytes(dtype, rows, cols, bias)


def reqat_layer_norm_backward(dy, lddy, x, ldx, dtype, rows, cols, weight, w_dtype, stats, center, dx, lddx, dweight,
                              dbias, workspace, stream):
    return load().reqat_layer_norm_backward(dy, lddy, x, ldx, dtype, rows, cols, weight, w_dtype, stats, center, dx, lddx,
                                            dweight, dbias, workspace, stream)


def reqat_embedding(ids, T, table, dtype, V, D, ld_table, scale, out, ldo, stream):
    return load().reqat_embedding(ids, T, table, dtype, V, D, ld_table, scale, out, ldo, stream)


def reqat_embedding_workspace_bytes(T, V, D) -> int:
    return load().reqat_embedding_workspace_bytes(T, V, D)


def reqat_embedding_backward(dy, dtype, lddy, ids, T, V, D, scale, dtable, table_dtype, ld_table, accumulate, workspace,
                             stream):
    return load().reqat_embedding_backward(dy, dtype, lddy, ids, T, V, D, scale, dtable, table_dtype, ld_table, accumulate,
                                           workspace, stream)


class AdamwTensor(ctypes.Structure):
    """reqat_adamw_tensor of the C ABI."""
    _fields_ = [("p", _VP), ("g", _VP), ("m", _VP), ("v", _VP), ("m_scale", _VP), ("v_scale", _VP), ("copy", _VP),
                ("n", _I64)]


class AdamwHyper(ctypes.Structure):
    """reqat_adamw_hyper of the C ABI."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("step", _I64)]


def reqat_adamw_step(tensors, count, p_dtype, g_dtype, state_bits, hyper, grad_scale, coef, stream):
    """tensors: an array of AdamwTensor, or its 8 words a tensor in an array.array (or None), hyper: an AdamwHyper (or
    None)."""
    at = tensors.buffer_info()[0] if isinstance(tensors, array.array) else _cache_ref(tensors)
    return load().reqat_adamw_step(at, count, p_dtype, g_dtype, state_bits, _cache_ref(hyper), grad_scale,
                                   coef, stream)


def reqat_adamw_coefficients(hyper, lr, step, coef, stream):
    return load().reqat_adamw_coefficients(_cache_ref(hyper), lr, step, coef, stream)


def reqat_adamw_moments(m, m_scale, v, v_scale, n, m_out, v_out, stream):
    return load().reqat_adamw_moments(m, m_scale, v, v_scale, n, m_out, v_out, stream)


def reqat_w4a4_packed_bytes(fmt, N, K) -> int:
    return load().reqat_w4a4_packed_bytes(fmt, N, K)


def reqat_pack_w4a4(fmt, w_codes, w_scales, N, K, packed, stream):
    return load().reqat_pack_w4a4(fmt, w_codes, w_scales, N, K, packed, stream)


def reqat_gemm_w4a4_packed(fmt, M, N, K, a_codes, a_scales, a_ts, packed, b_ts, y, y_dtype, ldy, stream):
    return load().reqat_gemm_w4a4_packed(fmt, M, N, K, a_codes, a_scales, a_ts, packed, b_ts, y, y_dtype, ldy,
                                         stream)


def reqat_linear_w4a4_packed(fmt, M, N, K, x, ldx, x_ts, ts, packed, w_ts, y, y_dtype, ldy, workspace, stream):
    return load().reqat_linear_w4a4_packed(fmt, M, N, K, x, ldx, x_ts, ts, packed, w_ts, y, y_dtype, ldy,
                                           workspace, stream)


def reqat_linear_workspace_bytes(fmt, M, K) -> int:
    return load().reqat_linear_workspace_bytes(fmt, M, K)


def reqat_linear_w4a4_noalloc(fmt, M, N, K, x, ldx, x_ts, ts, w_codes, w_scales, w_ts, y, y_dtype, ldy, stream):
    return load().reqat_linear_w4a4_noalloc(fmt, M, N, K, x, ldx, x_ts, ts, w_codes, w_scales, w_ts, y,
                                            y_dtype, ldy, stream)


def reqat_workspace_bytes() -> int:
    return load().reqat_workspace_bytes()


def reqat_status_str(s: int) -> str:
    return load().reqat_status_str(s).decode()


def reqat_abi_version() -> int:
    return load().reqat_abi_version()


# ------------------------------------------------------------------ torch conveniences

def _stream(device) -> int:
    """The handle of the device's current stream (without a Stream object around it: 3 us less per call)."""
    index = device.index
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if index is None else index)


def _check(st: int, where: str):
    if st != 0:
        raise ReqatError(st, where)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _x2d(x: torch.Tensor):
    if not isinstance(x, torch.Tensor) or x.dtype != torch.bfloat16 or x.dim() != 2:
        raise TypeError("expected a 2-D bfloat16 tensor")
    if x.stride(1) != 1:
        raise ValueError("rows must be contiguous")
    return x.shape[0], x.shape[1], x.stride(0)


def _same_device(t, device, name):
    if t.device != device:
        raise ValueError("%s must be on %s" % (name, device))


def _require_cuda(t, name="x"):
    """Checked after every shape, dtype and size check, right before the C call."""
    if not t.is_cuda:
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)


def _packed_u8(t, rows, cols, device, name):
    """A uint8 [rows, cols] tensor with dense rows (the C ABI takes no row stride for codes and scales)."""
    if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8:
        raise TypeError("%s must be a uint8 tensor" % name)
    if tuple(t.shape) != (rows, cols):
        raise ValueError("%s must have shape (%d, %d), got %s" % (name, rows, cols, tuple(t.shape)))
    if rows > 1 and cols > 0 and t.stride(0) != cols or cols > 1 and t.stride(1) != 1:
        raise ValueError("%s must be contiguous" % name)
    _same_device(t, device, name)
    return t


def _out2d(t, rows, cols, dtype, device, name):
    """An output [rows, cols] of `dtype` with unit column stride; returns its row stride."""
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError("%s must be a %s tensor" % (name, dtype))
    if t.dim() != 2 or tuple(t.shape) != (rows, cols):
        raise ValueError("%s must have shape (%d, %d), got %s" % (name, rows, cols, tuple(t.shape)))
    if cols > 1 and t.stride(1) != 1:
        raise ValueError("%s rows must be contiguous" % name)
    _same_device(t, device, name)
    return t.stride(0) if rows > 1 else max(cols, 1)


def _workspace_arg(ws, nbytes, device, name="ws"):
    if not isinstance(ws, torch.Tensor) or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise TypeError("%s must be a contiguous uint8 tensor" % name)
    if ws.numel() < nbytes:
        raise ValueError("%s holds %d bytes, %d needed" % (name, ws.numel(), nbytes))
    _same_device(ws, device, name)
    return ws


def _scale_arg(g, fmt, device, name):
    """The 1-element float32 device tensor of an NVFP4 global scale (MXFP4: None)."""
    if fmt == MXFP4:
        if g is not None:
            raise ValueError("MXFP4 has no global scale (%s must be None)" % name)
        return None
    if not isinstance(g, torch.Tensor) or g.dtype != torch.float32 or g.numel() < 1:
        raise TypeError("%s must be a float32 tensor holding the NVFP4 global scale" % name)
    _same_device(g, device, name)
    return g


def _fmt_arg(fmt):
    if fmt not in (NVFP4, MXFP4):
        raise ValueError("unknown format %r" % (fmt,))
    return fmt


_workspaces: dict = {}


def workspace(device) -> torch.Tensor:
    """A per-device workspace tensor (cached; calls on different streams must not share it)."""
    device = torch.device(device)
    key = (device.index if device.index is not None else torch.cuda.current_device())
    ws = _workspaces.get(key)
    if ws is None:
        ws = torch.empty(reqat_workspace_bytes(), dtype=torch.uint8, device=device)
        _workspaces[key] = ws
    return ws


def _gscale(fmt, x, tensor_scale, g_out=None):
    """(tensor_scale tensor or None, ts mode).  g_out: preallocated 1-element
    float32 tensor that receives the computed NVFP4 global scale."""
    if fmt == MXFP4:
        if tensor_scale is not None:
            raise ValueError("MXFP4 has no global scale")
        return None, TS_COMPUTE
    if tensor_scale is None:
        if g_out is not None:
            return _scale_arg(g_out, fmt, x.device, "g_out"), TS_COMPUTE
        return torch.empty(1, dtype=torch.float32, device=x.device), TS_COMPUTE
    if isinstance(tensor_scale, torch.Tensor):
        return _scale_arg(tensor_scale, fmt, x.device, "tensor_scale"), TS_GIVEN
    return torch.tensor([float(tensor_scale)], dtype=torch.float32, device=x.device), TS_GIVEN


def quantize(x: torch.Tensor, fmt: int = NVFP4, tensor_scale=None, out=None, g_out=None):
    """Quantize a 2-D bfloat16 CUDA tensor.  Returns (codes, scales, g) with g a
    1-element float32 tensor (NVFP4: computed unless given) or None (MXFP4)."""
    rows, cols, ldx = _x2d(x)
    B = BLOCK[_fmt_arg(fmt)]
    if cols % B:
        raise ValueError("cols must be a multiple of %d" % B)
    if out is not None:
        codes, scales = out
        _packed_u8(codes, rows, cols // 2, x.device, "codes")
        _packed_u8(scales, rows, cols // B, x.device, "scales")
    else:
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, cols // B), dtype=torch.uint8, device=x.device)
    g, ts = _gscale(fmt, x, tensor_scale, g_out)
    _require_cuda(x, 'x')
    ws = workspace(x.device)
    st = reqat_quantize_fp4(fmt, x.data_ptr(), rows, cols, ldx, codes.data_ptr(), scales.data_ptr(),
                            _ptr(g), ts, ws.data_ptr(), _stream(x.device))
    _check(st, "reqat_quantize_fp4")
    return codes, scales, g


def fakequant(x: torch.Tensor, fmt: int = NVFP4, tensor_scale=None, out=None, g_out=None):
    """Quantize-dequantize to bfloat16.  Returns (y, g)."""
    rows, cols, ldx = _x2d(x)
    _fmt_arg(fmt)
    y = out if out is not None else torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    ldy = _out2d(y, rows, cols, torch.bfloat16, x.device, "out")
    g, ts = _gscale(fmt, x, tensor_scale, g_out)
    _require_cuda(x, 'x')
    ws = workspace(x.device)
    st = reqat_fakequant_fp4(fmt, x.data_ptr(), rows, cols, ldx, y.data_ptr(), ldy, _ptr(g),
                             ts, ws.data_ptr(), _stream(x.device))
    _check(st, "reqat_fakequant_fp4")
    return y, g


def quantize_fakequant(x: torch.Tensor, fmt: int = NVFP4, tensor_scale=None, out=None, g_out=None):
    """Quantize and quantize-dequantize in one pass over x.  Returns
    (codes, scales, y, g): codes/scales as quantize(), y (bfloat16) as fakequant()."""
    rows, cols, ldx = _x2d(x)
    B = BLOCK[_fmt_arg(fmt)]
    if cols % B:
        raise ValueError("cols must be a multiple of %d" % B)
    if out is not None:
        codes, scales, y = out
        _packed_u8(codes, rows, cols // 2, x.device, "codes")
        _packed_u8(scales, rows, cols // B, x.device, "scales")
    else:
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, cols // B), dtype=torch.uint8, device=x.device)
        y = torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    ldy = _out2d(y, rows, cols, torch.bfloat16, x.device, "y")
    g, ts = _gscale(fmt, x, tensor_scale, g_out)
    _require_cuda(x, 'x')
    ws = workspace(x.device)
    st = reqat_quantize_fakequant_fp4(fmt, x.data_ptr(), rows, cols, ldx, codes.data_ptr(), scales.data_ptr(),
                                      y.data_ptr(), ldy, _ptr(g), ts, ws.data_ptr(), _stream(x.device))
    _check(st, "reqat_quantize_fakequant_fp4")
    return codes, scales, y, g


def quantize_rht(x: torch.Tensor, signs: int, out=None):
    """MXFP4 codes and scales of the block-rotated rows of x (randomized Hadamard
    of 32 with the given 32-bit sign draw).  Returns (codes, scales)."""
    rows, cols, ldx = _x2d(x)
    if cols % 32:
        raise ValueError("cols must be a multiple of 32")
    if out is not None:
        codes, scales = out
        _packed_u8(codes, rows, cols // 2, x.device, "codes")
        _packed_u8(scales, rows, cols // 32, x.device, "scales")
    else:
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, cols // 32), dtype=torch.uint8, device=x.device)
    _require_cuda(x, 'x')
    st = reqat_quantize_mxfp4_rht(x.data_ptr(), rows, cols, ldx, signs & 0xFFFFFFFF, codes.data_ptr(),
                                  scales.data_ptr(), _stream(x.device))
    _check(st, "reqat_quantize_mxfp4_rht")
    return codes, scales


def fakequant_rht(x: torch.Tensor, signs: int, out=None):
    """bfloat16 quantize-dequantize of the block-rotated rows (rotated basis)."""
    rows, cols, ldx = _x2d(x)
    y = out if out is not None else torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    ldy = _out2d(y, rows, cols, torch.bfloat16, x.device, "out")
    _require_cuda(x, 'x')
    st = reqat_fakequant_mxfp4_rht(x.data_ptr(), rows, cols, ldx, signs & 0xFFFFFFFF, y.data_ptr(),
                                   ldy, _stream(x.device))
    _check(st, "reqat_fakequant_mxfp4_rht")
    return y


def gemm(fmt, a_codes, a_scales, a_g, b_codes, b_scales, b_g, out_dtype=torch.float32, out=None):
    """Y[M, N] = A^ B^T with FP32 accumulation; Y float32 or bfloat16."""
    B = BLOCK[_fmt_arg(fmt)]
    dev = a_codes.device
    if a_codes.dim() != 2 or b_codes.dim() != 2:
        raise ValueError("codes must be 2-D")
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    N = b_codes.shape[0]
    if b_codes.shape[1] * 2 != K:
        raise ValueError("K mismatch")
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    _packed_u8(a_codes, M, K // 2, dev, "a_codes")
    _packed_u8(a_scales, M, K // B, dev, "a_scales")
    _packed_u8(b_codes, N, K // 2, dev, "b_codes")
    _packed_u8(b_scales, N, K // B, dev, "b_scales")
    _scale_arg(a_g, fmt, dev, "a_g")
    _scale_arg(b_g, fmt, dev, "b_g")
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=dev)
    ldy = _out2d(y, M, N, out_dtype, dev, "out")
    _require_cuda(a_codes, 'a_codes')
    st = reqat_gemm_w4a4(fmt, M, N, K, a_codes.data_ptr(), a_scales.data_ptr(), _ptr(a_g),
                         b_codes.data_ptr(), b_scales.data_ptr(), _ptr(b_g), y.data_ptr(), dt,
                         ldy, _stream(dev))
    _check(st, "reqat_gemm_w4a4")
    return y


def _dtype_arg(out_dtype):
    if out_dtype == torch.float32:
        return DT_F32
    if out_dtype == torch.bfloat16:
        return DT_BF16
    raise TypeError("out_dtype must be torch.float32 or torch.bfloat16")


def _shift_ptr(shift, cols, device):
    if shift is None:
        return None, None
    if shift.dtype != torch.float32 or shift.numel() != cols or not shift.is_contiguous() \
            or shift.device != device:
        raise ValueError("shift must be a contiguous float32 tensor of cols values on the same device")
    return shift, shift.data_ptr()


def quantize_kv4(x: torch.Tensor, shift=None, tensor_scale=None, out=None, g_out=None):
    """KV4 (E1M2 + E4M3 block scales of 16 + FP32 tensor scale) of x - shift.
    Returns (codes, scales, g)."""
    rows, cols, ldx = _x2d(x)
    if cols % 16:
        raise ValueError("cols must be a multiple of 16")
    if out is not None:
        codes, scales = out
        _packed_u8(codes, rows, cols // 2, x.device, "codes")
        _packed_u8(scales, rows, cols // 16, x.device, "scales")
    else:
        codes = torch.empty((rows, cols // 2), dtype=torch.uint8, device=x.device)
        scales = torch.empty((rows, cols // 16), dtype=torch.uint8, device=x.device)
    g, ts = _gscale(NVFP4, x, tensor_scale, g_out)
    _, sp = _shift_ptr(shift, cols, x.device)
    _require_cuda(x, 'x')
    st = reqat_quantize_kv4(x.data_ptr(), rows, cols, ldx, sp, codes.data_ptr(), scales.data_ptr(), _ptr(g), ts,
                            workspace(x.device).data_ptr(), _stream(x.device))
    _check(st, "reqat_quantize_kv4")
    return codes, scales, g


def fakequant_kv4(x: torch.Tensor, shift=None, tensor_scale=None, out=None, g_out=None):
    """bfloat16 quantize-dequantize of x - shift in KV4.  Returns (y, g)."""
    rows, cols, ldx = _x2d(x)
    y = out if out is not None else torch.empty((rows, cols), dtype=torch.bfloat16, device=x.device)
    ldy = _out2d(y, rows, cols, torch.bfloat16, x.device, "out")
    g, ts = _gscale(NVFP4, x, tensor_scale, g_out)
    _, sp = _shift_ptr(shift, cols, x.device)
    _require_cuda(x, 'x')
    st = reqat_fakequant_kv4(x.data_ptr(), rows, cols, ldx, sp, y.data_ptr(), ldy, _ptr(g), ts,
                             workspace(x.device).data_ptr(), _stream(x.device))
    _check(st, "reqat_fakequant_kv4")
    return y, g


class Kv4Cache:
    """A paged KV4 cache: ``num_pages`` pages of ``page_size`` tokens (a power of two, 16 or more) of ``kv_heads``
    heads of ``head_dim`` (64 or 128) channels, with the calibrated tensor scales of keys and values and, optionally,
    the post-RoPE shift of the keys (float32 [kv_heads * head_dim]).

    A scale is a number, or a float32 tensor of one element on the device.  The codes and scales (``k_codes``,
    ``k_scales``, ``v_codes``, ``v_scales``) have the layout that include/reqat.h states.  Which pages belong to which
    sequence is the caller's: a slot is page * page_size + the token's place in the page.  Scales, shift and arrays
    may be written in place or assigned; the sizes and the device stay."""

    _ARRAYS = {"k_codes": 2, "k_scales": 16, "v_codes": 2, "v_scales": 16}       # channels to a byte
    _SIZES = frozenset(("device", "num_pages", "page_size", "kv_heads", "head_dim", "width"))

    def __init__(self, num_pages, page_size, kv_heads, head_dim=128, k_scale=1.0, v_scale=1.0, k_shift=None,
                 device="cuda"):
        if num_pages < 0 or kv_heads < 1:
            raise ValueError("num_pages must be >= 0 and kv_heads >= 1")
        if page_size < 16 or page_size > 1 << 20 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two from 16 to 2^20")
        if head_dim not in (64, 128):
            raise ValueError("head_dim must be 64 or 128")
        self.device = torch.device(device)
        if self.device.type == "cuda" and self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.num_pages, self.page_size, self.kv_heads, self.head_dim = num_pages, page_size, kv_heads, head_dim
        self.width = kv_heads * head_dim         # channels of a token's keys, and of its values

        self.k_scale, self.v_scale, self.k_shift = k_scale, v_scale, k_shift
        for name in self._ARRAYS:
            setattr(self, name, torch.zeros(self._bytes(name), dtype=torch.uint8, device=self.device))

    def _bytes(self, name):
        return self.num_pages * self.page_size * self.width // self._ARRAYS[name]

    def _checked(self, name, value):
        if name == "k_shift":
            return _shift_ptr(value, self.width, self.device)[0]
        if name in self._ARRAYS:
            return _index_arg(value, (self._bytes(name),), torch.uint8, self.device, name)
        if isinstance(value, torch.Tensor):
            return _scale_arg(value, NVFP4, self.device, name)
        g = torch.tensor([float(value)], dtype=torch.float32)
        if not 0.0 < float(g) < float("inf"):
            raise ValueError("%s must be a positive, finite FP32 number" % name)
        return g.to(self.device)

    def __setattr__(self, name, value):
        if name in self._ARRAYS or name in ("k_scale", "v_scale", "k_shift"):
            value = self._checked(name, value)
            self.__dict__.pop("struct", None)            # it has the old tensor's address
        elif name in self._SIZES and name in self.__dict__:
            raise AttributeError("%s of a Kv4Cache does not change" % name)
        object.__setattr__(self, name, value)

    def __getstate__(self):
        return {name: value for name, value in self.__dict__.items() if name != "struct"}

    @functools.cached_property
    def struct(self) -> Kv4CacheStruct:
        """reqat_kv4_cache of this cache, until one of its tensors is replaced."""
        return Kv4CacheStruct(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(),
                              self.v_scales.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(),
                              _ptr(self.k_shift), self.num_pages, self.page_size, self.kv_heads, self.head_dim)


def _cache_arg(cache):
    if not isinstance(cache, Kv4Cache):
        raise TypeError("cache must be a Kv4Cache")
    return cache


def _index_arg(t, shape, dtype, device, name):
    """A contiguous tensor that the kernels read on the device (the whole check first: decode steps are short)."""
    if type(t) is torch.Tensor and t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return t
    if not isinstance(t, torch.Tensor) or t.dtype != dtype:
        raise TypeError("%s must be a %s tensor" % (name, dtype))
    if tuple(t.shape) != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, shape, tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    _same_device(t, device, name)
    return t


def _rows_arg(x, rows, cols, device, name):
    """A bfloat16 [rows, cols] tensor, rows possibly strided; returns its row stride."""
    if type(x) is torch.Tensor and x.dtype is torch.bfloat16 and x.shape == (rows, cols) and x.device == device:
        ld, one = x.stride()
        if one == 1:
            return ld if rows > 1 else max(cols, 1)
    if not isinstance(x, torch.Tensor) or x.dtype != torch.bfloat16 or x.dim() != 2:
        raise TypeError("%s must be a 2-D bfloat16 tensor" % name)
    return _out2d(x, rows, cols, torch.bfloat16, device, name)


def kv4_append(cache, k, v, slots, q=None, rope=None, positions=None, q_out=None):
    """Write T tokens into a Kv4Cache in one pass: keys k and values v (bfloat16 [T, kv_heads * head_dim], rows may
    be strided) go to ``slots`` (int64 [T]; a slot outside the cache, such as -1, marks padding), keys rotated when
    ``rope`` = (cos, sin), float32 [P, head_dim / 2], and ``positions`` (int32 [T]) are given, then less the cache's
    shift.  Queries q [T, q_heads * head_dim] are rotated too; returns them (into q_out when given; q itself is
    allowed), or None without q."""
    _cache_arg(cache)
    dev, D = cache.device, cache.head_dim
    T = k.shape[0] if isinstance(k, torch.Tensor) and k.dim() == 2 else 0
    ldk, ldv = _rows_arg(k, T, cache.width, dev, "k"), _rows_arg(v, T, cache.width, dev, "v")
    _index_arg(slots, (T,), torch.int64, dev, "slots")
    cos = sin = None
    rope_len = 0
    if rope is not None:
        cos, sin = rope
        if not isinstance(cos, torch.Tensor) or cos.dim() != 2:
            raise TypeError("rope must be two float32 tensors [P, head_dim / 2]")
        rope_len = cos.shape[0]
        _index_arg(cos, (rope_len, D // 2), torch.float32, dev, "rope cos")
        _index_arg(sin, (rope_len, D // 2), torch.float32, dev, "rope sin")
        _index_arg(positions, (T,), torch.int32, dev, "positions")
    elif positions is not None:
        raise ValueError("positions without rope")
    ldq = ldqo = q_heads = 0
    if q is not None:
        if rope is None:
            raise ValueError("queries are rotated: q needs rope and positions")
        if not isinstance(q, torch.Tensor) or q.dim() != 2 or q.shape[1] == 0 or q.shape[1] % D:
            raise ValueError("q must be [T, q_heads * head_dim]")
        q_heads = q.shape[1] // D
        ldq = _rows_arg(q, T, q.shape[1], dev, "q")
        if q_out is None:
            q_out = torch.empty((T, q.shape[1]), dtype=torch.bfloat16, device=dev)
        ldqo = _rows_arg(q_out, T, q.shape[1], dev, "q_out")
    elif q_out is not None:
        raise ValueError("q_out without q")
    _require_cuda(k, "k")
    st = reqat_kv4_append(cache.struct, T, slots.data_ptr(), k.data_ptr(), ldk, v.data_ptr(), ldv, _ptr(q), ldq, q_heads,
                          _ptr(q_out), ldqo, _ptr(cos), _ptr(sin), _ptr(positions), rope_len, _stream(dev))
    _check(st, "reqat_kv4_append")
    return q_out


def kv4_gather(cache, slots, add_shift=False, out=None):
    """The keys and values that ``slots`` (int64 [T]) of a Kv4Cache hold, as bfloat16 [T, kv_heads * head_dim] each
    (zeros for a slot outside the cache); keys in the shifted domain, or with the shift added.  out: (k, v)
    preallocated, rows may be strided."""
    _cache_arg(cache)
    if not isinstance(slots, torch.Tensor) or slots.dim() != 1:
        raise TypeError("slots must be a 1-D int64 tensor")
    T, dev = slots.shape[0], cache.device
    _index_arg(slots, (T,), torch.int64, dev, "slots")
    if out is None:
        out = torch.empty((2, T, cache.width), dtype=torch.bfloat16, device=dev).unbind(0)
    k, v = out
    ldk = _rows_arg(k, T, cache.width, dev, "out[0]")
    ldv = _rows_arg(v, T, cache.width, dev, "out[1]")
    _require_cuda(slots, "slots")
    st = reqat_kv4_gather(cache.struct, T, slots.data_ptr(), k.data_ptr(), ldk, v.data_ptr(), ldv, 1 if add_shift else 0,
                          _stream(dev))
    _check(st, "reqat_kv4_gather")
    return k, v


@functools.lru_cache(maxsize=1024)
def _kv4_workspace(B, T, max_q, max_kv, q_heads, kv_heads, head_dim) -> int:
    return reqat_kv4_attention_workspace_bytes(B, T, max_q, max_kv, q_heads, kv_heads, head_dim)


def kv4_attention(q, cache, block_table, kv_len, q_start=None, max_q=None, max_kv=None, causal=True, sm_scale=None,
                  out=None, return_lse=False, ws=None):
    """Attention of the queries of B sequences over their tokens in a Kv4Cache.

    q: bfloat16 [T, q_heads * head_dim] (rows may be strided); block_table: int32 [B, pages of a sequence];
    kv_len: int32 [B], cached tokens, the new ones included; q_start: int32 [B + 1], the first query row of each
    sequence, or None: one query each.  max_q and max_kv bound the queries and tokens of every sequence on the host
    (by default T, 1 without q_start, and what the table can hold); closer bounds launch less.  causal: the queries
    are the last tokens of their sequence.  sm_scale: default head_dim ** -0.5.  ws: uint8 tensor of at least
    reqat_kv4_attention_workspace_bytes(B, T, max_q, max_kv, q_heads, kv_heads, head_dim) bytes; one of the largest
    sizes serves every smaller call.
    Returns out, bfloat16 like q, or (out, lse) with lse float32 [T, q_heads]."""
    _cache_arg(cache)
    dev, D = cache.device, cache.head_dim
    if not isinstance(q, torch.Tensor) or q.dim() != 2 or q.shape[1] == 0 or q.shape[1] % cache.width:
        raise ValueError("q must be [T, q_heads * head_dim], q_heads a multiple of kv_heads")
    T, q_heads = q.shape[0], q.shape[1] // D
    ldq = _rows_arg(q, T, q.shape[1], dev, "q")
    if not isinstance(block_table, torch.Tensor) or block_table.dtype != torch.int32 or block_table.dim() != 2:
        raise TypeError("block_table must be a 2-D int32 tensor")
    B, cols = block_table.shape
    if cols > 1 and block_table.stride(1) != 1 or B > 1 and block_table.stride(0) < cols:
        raise ValueError("block_table rows must be contiguous")
    ld_table = block_table.stride(0) if B > 1 else cols
    _same_device(block_table, dev, "block_table")
    _index_arg(kv_len, (B,), torch.int32, dev, "kv_len")
    if q_start is not None:
        _index_arg(q_start, (B + 1,), torch.int32, dev, "q_start")
    elif T != B:
        raise ValueError("without q_start there is one query per sequence")
    if max_q is None:
        max_q = T if q_start is not None else 1
    if max_kv is None:
        max_kv = min(cols * cache.page_size, 1 << 30)
    if sm_scale is None:
        sm_scale = D ** -0.5
    y = out if out is not None else torch.empty((T, q.shape[1]), dtype=torch.bfloat16, device=dev)
    ldo = _rows_arg(y, T, q.shape[1], dev, "out")
    lse = torch.empty((T, q_heads), dtype=torch.float32, device=dev) if return_lse else None
    need = _kv4_workspace(B, T, max_q, max_kv, q_heads, cache.kv_heads, D)
    if ws is not None:
        _workspace_arg(ws, need, dev)
    _require_cuda(q, "q")
    if ws is None and need > 0:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    st = reqat_kv4_attention(cache.struct, B, T, q.data_ptr(), ldq, q_heads, _ptr(q_start), kv_len.data_ptr(),
                             block_table.data_ptr(), ld_table, cols, max_q, max_kv, 1 if causal else 0, sm_scale,
                             y.data_ptr(), ldo, _ptr(lse), _ptr(ws) if need > 0 else None, _stream(dev))
    _check(st, "reqat_kv4_attention")
    return (y, lse) if return_lse else y


def gemm_w4a16(x: torch.Tensor, w_codes, w_scales, out_dtype=torch.float32, out=None, ws=None):
    """Y = x . W^T with x bfloat16 [M, K] and MXFP4 weights (codes [N, K/2],
    scales [N, K/32]) dequantized to bfloat16; FP32 accumulation.
    ws: optional workspace tensor of reqat_w4a16_workspace_bytes(M, N, K) bytes."""
    M, K, ldx = _x2d(x)
    if w_codes.dim() != 2:
        raise ValueError("w_codes must be 2-D")
    N = w_codes.shape[0]
    if w_codes.shape[1] * 2 != K:
        raise ValueError("K mismatch")
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    _packed_u8(w_codes, N, K // 2, x.device, "w_codes")
    _packed_u8(w_scales, N, K // 32, x.device, "w_scales")
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=x.device)
    ldy = _out2d(y, M, N, out_dtype, x.device, "out")
    nbytes = reqat_w4a16_workspace_bytes(M, N, K)
    if ws is None and nbytes:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    if ws is not None:
        _workspace_arg(ws, nbytes, x.device)
    _require_cuda(x, 'x')
    st = reqat_gemm_w4a16(M, N, K, x.data_ptr(), ldx, w_codes.data_ptr(), w_scales.data_ptr(), y.data_ptr(),
                          dt, ldy, _ptr(ws), _stream(x.device))
    _check(st, "reqat_gemm_w4a16")
    return y


def pack_w4a16(w_codes, w_scales, out=None):
    """Packed weight image of MXFP4 weights (codes [N, K/2], scales [N, K/32])
    for gemm_w4a16_packed: a uint8 tensor of reqat_w4a16_packed_bytes(N, K)."""
    if w_codes.dim() != 2:
        raise ValueError("w_codes must be 2-D")
    N, K = w_codes.shape[0], w_codes.shape[1] * 2
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    _packed_u8(w_codes, N, K // 2, w_codes.device, "w_codes")
    _packed_u8(w_scales, N, K // 32, w_codes.device, "w_scales")
    nbytes = reqat_w4a16_packed_bytes(N, K)
    packed = out if out is not None else torch.empty(max(nbytes, 16), dtype=torch.uint8, device=w_codes.device)
    if packed.dtype != torch.uint8 or not packed.is_contiguous() or packed.numel() < nbytes \
            or packed.device != w_codes.device:
        raise ValueError("out must be a contiguous uint8 tensor of at least %d bytes on the weights' device" % nbytes)
    _require_cuda(w_codes, "w_codes")
    st = reqat_pack_w4a16(w_codes.data_ptr(), w_scales.data_ptr(), N, K, packed.data_ptr(), _stream(w_codes.device))
    _check(st, "reqat_pack_w4a16")
    return packed


def gemm_w4a16_packed(x: torch.Tensor, packed, N, out_dtype=torch.float32, out=None, ws=None):
    """gemm_w4a16 on the packed image (pack_w4a16) of N x K weights: same result, bit for bit."""
    M, K, ldx = _x2d(x)
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    nbytes_w = reqat_w4a16_packed_bytes(N, K)
    if packed.dtype != torch.uint8 or not packed.is_contiguous() or packed.numel() < nbytes_w \
            or packed.device != x.device:
        raise ValueError("packed must be the contiguous uint8 image of %d bytes on x's device" % nbytes_w)
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=x.device)
    ldy = _out2d(y, M, N, out_dtype, x.device, "out")
    nbytes = reqat_w4a16_workspace_bytes(M, N, K)
    if ws is None and nbytes:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    if ws is not None:
        _workspace_arg(ws, nbytes, x.device)
    _require_cuda(x, 'x')
    st = reqat_gemm_w4a16_packed(M, N, K, x.data_ptr(), ldx, packed.data_ptr(), y.data_ptr(), dt, ldy, _ptr(ws),
                                 _stream(x.device))
    _check(st, "reqat_gemm_w4a16_packed")
    return y


def linear(x: torch.Tensor, fmt, w_codes, w_scales, w_g, x_tensor_scale=None, out_dtype=torch.bfloat16,
           out=None, g_out=None, ws=None):
    """Y = quantize(x) . W^T for already-quantized weights.  Returns (Y, g_x).
    ws: optional workspace tensor of reqat_linear_workspace_bytes(fmt, M, K) bytes."""
    M, K, ldx = _x2d(x)
    B = BLOCK[_fmt_arg(fmt)]
    if w_codes.dim() != 2:
        raise ValueError("w_codes must be 2-D")
    N = w_codes.shape[0]
    if w_codes.shape[1] * 2 != K:
        raise ValueError("K mismatch")
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    _packed_u8(w_codes, N, K // 2, x.device, "w_codes")
    _packed_u8(w_scales, N, K // B, x.device, "w_scales")
    _scale_arg(w_g, fmt, x.device, "w_g")
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=x.device)
    ldy = _out2d(y, M, N, out_dtype, x.device, "out")
    g, ts = _gscale(fmt, x, x_tensor_scale, g_out)
    nbytes = reqat_linear_workspace_bytes(fmt, M, K)
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    _workspace_arg(ws, nbytes, x.device)
    _require_cuda(x, 'x')
    st = reqat_linear_w4a4(fmt, M, N, K, x.data_ptr(), ldx, _ptr(g), ts, w_codes.data_ptr(),
                           w_scales.data_ptr(), _ptr(w_g), y.data_ptr(), dt, ldy, ws.data_ptr(),
                           _stream(x.device))
    _check(st, "reqat_linear_w4a4")
    return y, g


def pack_w4a4(w_codes, w_scales, fmt, out=None):
    """Packed decode image of W4A4 weights (codes [N, K/2], scales [N, K/B]) for
    gemm_packed / linear_packed: a uint8 tensor of reqat_w4a4_packed_bytes(fmt, N, K)."""
    B = BLOCK[_fmt_arg(fmt)]
    if w_codes.dim() != 2:
        raise ValueError("w_codes must be 2-D")
    N, K = w_codes.shape[0], w_codes.shape[1] * 2
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    _packed_u8(w_codes, N, K // 2, w_codes.device, "w_codes")
    _packed_u8(w_scales, N, K // B, w_codes.device, "w_scales")
    nbytes = reqat_w4a4_packed_bytes(fmt, N, K)
    packed = out if out is not None else torch.empty(max(nbytes, 16), dtype=torch.uint8, device=w_codes.device)
    _packed_image_arg(packed, nbytes, w_codes.device, "out")
    _require_cuda(w_codes, "w_codes")
    st = reqat_pack_w4a4(fmt, w_codes.data_ptr(), w_scales.data_ptr(), N, K, packed.data_ptr(),
                         _stream(w_codes.device))
    _check(st, "reqat_pack_w4a4")
    return packed


def _packed_image_arg(packed, nbytes, device, name):
    if not isinstance(packed, torch.Tensor) or packed.dtype != torch.uint8 or not packed.is_contiguous() \
            or packed.numel() < nbytes or packed.device != device:
        raise ValueError("%s must be a contiguous uint8 tensor of at least %d bytes on %s" % (name, nbytes, device))


def gemm_packed(fmt, a_codes, a_scales, a_g, packed, N, b_g, out_dtype=torch.float32, out=None):
    """gemm() for M <= 64 on the packed image (pack_w4a4) of N x K weights: same result, bit for bit."""
    B = BLOCK[_fmt_arg(fmt)]
    dev = a_codes.device
    if a_codes.dim() != 2:
        raise ValueError("codes must be 2-D")
    M, K = a_codes.shape[0], a_codes.shape[1] * 2
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    if M > 64:
        raise ValueError("the packed image serves products with M <= 64")
    _packed_u8(a_codes, M, K // 2, dev, "a_codes")
    _packed_u8(a_scales, M, K // B, dev, "a_scales")
    _packed_image_arg(packed, reqat_w4a4_packed_bytes(fmt, N, K), dev, "packed")
    _scale_arg(a_g, fmt, dev, "a_g")
    _scale_arg(b_g, fmt, dev, "b_g")
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=dev)
    ldy = _out2d(y, M, N, out_dtype, dev, "out")
    _require_cuda(a_codes, 'a_codes')
    st = reqat_gemm_w4a4_packed(fmt, M, N, K, a_codes.data_ptr(), a_scales.data_ptr(), _ptr(a_g), packed.data_ptr(),
                                _ptr(b_g), y.data_ptr(), dt, ldy, _stream(dev))
    _check(st, "reqat_gemm_w4a4_packed")
    return y


def linear_packed(x: torch.Tensor, fmt, packed, N, w_g, x_tensor_scale=None, out_dtype=torch.bfloat16,
                  out=None, g_out=None, ws=None):
    """linear() for M <= 64 on the packed image (pack_w4a4) of N x K weights.  Returns (Y, g_x)."""
    M, K, ldx = _x2d(x)
    _fmt_arg(fmt)
    if K % 128:
        raise ValueError("K must be a multiple of 128")
    if M > 64:
        raise ValueError("the packed image serves products with M <= 64")
    _packed_image_arg(packed, reqat_w4a4_packed_bytes(fmt, N, K), x.device, "packed")
    _scale_arg(w_g, fmt, x.device, "w_g")
    dt = _dtype_arg(out_dtype)
    y = out if out is not None else torch.empty((M, N), dtype=out_dtype, device=x.device)
    ldy = _out2d(y, M, N, out_dtype, x.device, "out")
    g, ts = _gscale(fmt, x, x_tensor_scale, g_out)
    nbytes = reqat_linear_workspace_bytes(fmt, M, K)
    if ws is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device)
    _workspace_arg(ws, nbytes, x.device)
    _require_cuda(x, 'x')
    st = reqat_linear_w4a4_packed(fmt, M, N, K, x.data_ptr(), ldx, _ptr(g), ts, packed.data_ptr(), _ptr(w_g),
                                  y.data_ptr(), dt, ldy, ws.data_ptr(), _stream(x.device))
    _check(st, "reqat_linear_w4a4_packed")
    return y, g


def linear_workspace_views(ws: torch.Tensor, fmt, M: int, K: int):
    """(codes [M, K/2], scales [M, K/B]) views of the activation codes and scales
    that linear() leaves in its workspace: [4096 partial maxima | codes | scales | ...],
    each part on a 256-byte boundary."""
    B = BLOCK[_fmt_arg(fmt)]
    r256 = lambda n: (n + 255) // 256 * 256
    off = r256(4 * 4096)
    off2 = off + r256(M * (K // 2))
    codes = ws[off:off + M * (K // 2)].view(M, K // 2)
    scales = ws[off2:off2 + M * (K // B)].view(M, K // B)
    return codes, scales


# ------------------------------------------------------------------ QAT training side

def sem_loss(logits: torch.Tensor, targets: torch.Tensor, lam: float, eps: float = 1e-6):
    """SEM loss of bfloat16 logits [T, V] and int32 targets [T].  Returns
    (loss[4] = L, mean NLL, mean w H, tau; stats [T, 4]; weights [T])."""
    T, V, ld = _x2d(logits)
    if targets.dtype != torch.int32 or targets.numel() != T or not targets.is_contiguous():
        raise TypeError("targets must be a contiguous int32 tensor of T entries")
    stats = torch.empty((T, 4), dtype=torch.float32, device=logits.device)
    weights = torch.empty(T, dtype=torch.float32, device=logits.device)
    loss = torch.zeros(4, dtype=torch.float32, device=logits.device)
    _require_cuda(logits, 'logits')
    st = reqat_sem_loss(logits.data_ptr(), T, V, ld, targets.data_ptr(), lam, eps, stats.data_ptr(),
                        weights.data_ptr(), loss.data_ptr(), _stream(logits.device))
    _check(st, "reqat_sem_loss")
    return loss, stats, weights


def sem_loss_backward(logits, targets, stats, weights, lam: float, scale: float = 1.0, out_dtype=torch.bfloat16,
                      out=None):
    """dL/dlogits (weights held fixed) as out_dtype [T, V]."""
    T, V, ld = _x2d(logits)
    dt = _dtype_arg(out_dtype)
    if targets.dtype != torch.int32 or targets.numel() != T or not targets.is_contiguous():
        raise TypeError("targets must be a contiguous int32 tensor of T entries")
    for name, t, n in (("stats", stats, 4 * T), ("weights", weights, T)):
        if t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
            raise TypeError("%s must be a contiguous float32 tensor of %d entries" % (name, n))
        _same_device(t, logits.device, name)
    g = out if out is not None else torch.empty((T, V), dtype=out_dtype, device=logits.device)
    ldg = _out2d(g, T, V, out_dtype, logits.device, "out")
    _require_cuda(logits, 'logits')
    st = reqat_sem_loss_backward(logits.data_ptr(), T, V, ld, targets.data_ptr(), stats.data_ptr(),
                                 weights.data_ptr(), lam, scale, g.data_ptr(), dt, ldg,
                                 _stream(logits.device))
    _check(st, "reqat_sem_loss_backward")
    return g


class FakeQuantSTE(torch.autograd.Function):
    """QAT forward = fake-quant (bfloat16 in, bfloat16 out); backward = the
    straight-through estimator.  Under the ceil scale rules no element clips,
    so the estimator is the identity on the incoming gradient."""

    @staticmethod
    def forward(ctx, x, fmt=NVFP4):
        y, _ = fakequant(x.contiguous(), fmt)
        return y

    @staticmethod
    def backward(ctx, gy):
        return gy, None


class _Once(torch.autograd.Function):
    """Gradients of a kernel as functions of the tensors that they depend on, without a derivative of their own."""

    @staticmethod
    def forward(ctx, name, count, *tensors):
        ctx.name = name
        return tuple(t.view_as(t) for t in tensors[:count])

    @staticmethod
    def backward(ctx, *g):
        raise RuntimeError("%s has no second derivative" % ctx.name)


def _once(name, grads, *depends):
    """The gradients that a backward pass returns.  Under create_graph they are tied to what they were computed from, so that
    a derivative of them is refused; they would count as constants, and it would silently lack their part."""
    if not torch.is_grad_enabled():
        return grads
    new = [t for t in grads if t is not None]
    tied = iter(_Once.apply(name, len(new), *new, *depends))
    return tuple(None if t is None else next(tied) for t in grads)


class SemLoss(torch.autograd.Function):
    """The SEM loss as an autograd function over bfloat16 logits."""

    @staticmethod
    def forward(ctx, logits, targets, lam, eps=1e-6):
        loss, stats, weights = sem_loss(logits, targets, lam, eps)
        ctx.save_for_backward(logits, targets, stats, weights)
        ctx.lam = lam
        return loss[0]

    @staticmethod
    def backward(ctx, g):
        logits, targets, stats, weights = ctx.saved_tensors
        grad = sem_loss_backward(logits, targets, stats, weights, ctx.lam, scale=float(g.detach()), out_dtype=logits.dtype)
        return _once("SemLoss", (grad,), g, logits) + (None,) * 3


# ------------------------------------------------------------------ the operators around the quantized layers

def _call(fn, device, *args):
    """The C call with the device current, on its current stream."""
    current = torch.cuda.current_device()
    if device.index is None or device.index == current:
        st = fn(*args, torch._C._cuda_getCurrentRawStream(current))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream(device))
    _check(st, fn.__name__)


_FLOATS = {torch.bfloat16: DT_BF16, torch.float32: DT_F32}


def _float_rows(x, name):
    """Rows, columns, row stride and C dtype of a 2-D bfloat16 or float32 tensor with contiguous rows."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2 or x.dtype not in _FLOATS:
        raise TypeError("%s must be a 2-D bfloat16 or float32 tensor" % name)
    rows, cols = x.shape
    ld, one = x.stride()
    if cols > 1 and one != 1 or rows > 1 and ld < cols:
        raise ValueError("%s must have contiguous rows that do not overlap" % name)
    return rows, cols, ld if rows > 1 else max(cols, 1), _FLOATS[x.dtype]


def _float_out(t, rows, cols, dtype, device, name):
    """A given output [rows, cols], or a new one; returns it and its row stride."""
    if t is None:
        return torch.empty((rows, cols), dtype=dtype, device=device), max(cols, 1)
    ld = _out2d(t, rows, cols, dtype, device, name)
    if ld < cols:
        raise ValueError("%s must have rows that do not overlap" % name)
    return t, ld


def _written(*given):
    """Tells autograd that a caller's tensors hold something else now: a graph that keeps one refuses its backward pass."""
    torch.autograd.graph.increment_version(given)


def _vector(t, n, device, name, dtypes=(torch.float32,)):
    """A contiguous vector of n numbers (the whole check first: small calls are short)."""
    if isinstance(t, torch.Tensor) and t.dtype in dtypes and t.shape == (n,) and t.device == device and t.is_contiguous():
        return t
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
        raise TypeError("%s must be a tensor of %s" % (name, " or ".join(str(d) for d in dtypes)))
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError("%s must be contiguous, of shape (%d,), got %s" % (name, n, tuple(t.shape)))
    _same_device(t, device, name)
    return t


@functools.lru_cache(maxsize=1024)
def _policy_workspace(dtype, T, V) -> int:
    return reqat_policy_loss_workspace_bytes(dtype, T, V)


@functools.lru_cache(maxsize=1024)
def _norm_workspace(dtype, rows, cols, bias) -> int:
    return reqat_layer_norm_workspace_bytes(dtype, rows, cols, bias)


@functools.lru_cache(maxsize=1024)
def _embedding_workspace(T, V, D) -> int:
    return reqat_embedding_workspace_bytes(T, V, D)


def _policy_loss(logits, targets, old_logp, advantages, ref_logp, weights, clip_low, clip_high, kl_coef, temperature, grad,
                 out):
    T, V, ld, dt = _float_rows(logits, "logits")
    dev = logits.device
    _vector(targets, T, dev, "targets", (torch.int32,))
    _vector(old_logp, T, dev, "old_logp")
    _vector(advantages, T, dev, "advantages")
    if ref_logp is not None:
        _vector(ref_logp, T, dev, "ref_logp")
    elif kl_coef != 0.0:
        raise ValueError("kl_coef without ref_logp")
    if weights is not None:
        _vector(weights, T, dev, "weights")
    ldg, given = 0, out
    if grad:
        out, ldg = _float_out(out, T, V, logits.dtype, dev, "out")
    _require_cuda(logits, "logits")
    stats = torch.empty((T, 4), dtype=torch.float32, device=dev)
    loss = torch.empty(4, dtype=torch.float32, device=dev)
    need = _policy_workspace(dt, T, V)
    ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    _call(reqat_policy_loss, dev, logits.data_ptr(), dt, T, V, ld, targets.data_ptr(), old_logp.data_ptr(),
          advantages.data_ptr(), _ptr(ref_logp), _ptr(weights), clip_low, clip_high, kl_coef, temperature, stats.data_ptr(),
          loss.data_ptr(), _ptr(out) if grad else None, ldg, _ptr(ws))
    if given is not None:
        _written(given)
    return loss, stats, out


def policy_loss(logits, targets, old_logp, advantages, ref_logp=None, weights=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0, temperature=1.0):
    """Clipped policy loss with a KL term, of bfloat16 or float32 logits [T, V] (rows may be strided) and int32 targets,
    float32 old_logp, advantages, ref_logp and weights [T].

    With r = exp(log p - old_logp) and x = ref_logp - log p a token's loss is
    -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (exp(x) - x - 1); the loss is their sum under ``weights``
    (mask and normaliser in one, default 1 / T).  Rows of weight 0 are not read.  Returns (loss[4] = the loss, its
    surrogate part, the KL term's weighted sum, the clipped share; stats [T, 4] = log p of the target, log-sum-exp,
    dL / d log p, r)."""
    return _policy_loss(logits, targets, old_logp, advantages, ref_logp, weights, clip_low, clip_high, kl_coef, temperature,
                        False, None)[:2]


def policy_loss_grad(logits, targets, old_logp, advantages, ref_logp=None, weights=None, clip_low=0.2, clip_high=0.2,
                     kl_coef=0.0, temperature=1.0, out=None):
    """policy_loss() and dL/dlogits in one pass.  Returns (loss, stats, grad), grad like the logits; out: where it goes,
    the logits themselves allowed."""
    return _policy_loss(logits, targets, old_logp, advantages, ref_logp, weights, clip_low, clip_high, kl_coef, temperature,
                        True, out)


def policy_loss_backward(logits, targets, stats, temperature=1.0, grad_loss=None, out=None):
    """dL/dlogits from the logits and the statistics of policy_loss(), times grad_loss (a float32 tensor of one element).
    out may be the logits."""
    T, V, ld, dt = _float_rows(logits, "logits")
    dev = logits.device
    _vector(targets, T, dev, "targets", (torch.int32,))
    _index_arg(stats, (T, 4), torch.float32, dev, "stats")
    if grad_loss is not None:
        _scale_arg(grad_loss, NVFP4, dev, "grad_loss")
    given = out
    out, ldg = _float_out(out, T, V, logits.dtype, dev, "out")
    _require_cuda(logits, "logits")
    _call(reqat_policy_loss_backward, dev, logits.data_ptr(), dt, T, V, ld, targets.data_ptr(), stats.data_ptr(),
          temperature, _ptr(grad_loss), out.data_ptr(), ldg)
    if given is not None:
        _written(given)
    return out


def layer_norm(x, weight, bias=None, eps=1e-6, center=True, out=None):
    """Layer norm of the rows of x (bfloat16 or float32 [rows, cols], rows may be strided), or with center=False the
    root-mean-square norm, with weight and bias [cols] (bfloat16 or float32, both alike).  Returns (y like x; stats
    [rows, 2] = mean, 1 / standard deviation).  out may be x."""
    rows, cols, ldx, dt = _float_rows(x, "x")
    dev = x.device
    _vector(weight, cols, dev, "weight", _FLOATS)
    if bias is not None:
        _vector(bias, cols, dev, "bias", (weight.dtype,))
    y, ldy = _float_out(out, rows, cols, x.dtype, dev, "out")
    stats = torch.empty((rows, 2), dtype=torch.float32, device=dev)
    _require_cuda(x, "x")
    _call(reqat_layer_norm, dev, x.data_ptr(), dt, rows, cols, ldx, weight.data_ptr(), _ptr(bias), _dtype_arg(weight.dtype),
          eps, 1 if center else 0, y.data_ptr(), ldy, stats.data_ptr())
    if out is not None:
        _written(out)
    return y, stats


def layer_norm_backward(dy, x, weight, stats, center=True, bias=False, out=None, ws=None):
    """Gradients of layer_norm() from its input and statistics.  Returns (dx like x, dweight like weight, dbias or None).
    out (where dx goes) may be dy or x; ws: uint8 tensor of at least
    reqat_layer_norm_workspace_bytes(dtype, rows, cols, bias) bytes."""
    rows, cols, ldx, dt = _float_rows(x, "x")
    dev = x.device
    if not isinstance(dy, torch.Tensor) or dy.dtype != x.dtype or dy.shape != x.shape:
        raise ValueError("dy must have x's type and shape")
    lddy = _float_rows(dy, "dy")[2]
    _same_device(dy, dev, "dy")
    _vector(weight, cols, dev, "weight", _FLOATS)
    _index_arg(stats, (rows, 2), torch.float32, dev, "stats")
    dx, lddx = _float_out(out, rows, cols, x.dtype, dev, "out")
    need = _norm_workspace(dt, rows, cols, 1 if bias else 0)
    if ws is not None:
        _workspace_arg(ws, need, dev)
    _require_cuda(x, "x")
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    dw = torch.empty(cols, dtype=weight.dtype, device=dev)
    db = torch.empty(cols, dtype=weight.dtype, device=dev) if bias else None
    _call(reqat_layer_norm_backward, dev, dy.data_ptr(), lddy, x.data_ptr(), ldx, dt, rows, cols, weight.data_ptr(),
          _dtype_arg(weight.dtype), stats.data_ptr(), 1 if center else 0, dx.data_ptr(), lddx, dw.data_ptr(), _ptr(db),
          ws.data_ptr())
    if out is not None:
        _written(out)
    return dx, dw, db


def embedding(ids, table, scale=1.0, out=None):
    """Rows of the table (bfloat16 or float32 [V, D]) times scale, for int32 ids [T]: [T, D] like the table.  An id outside
    the table is padding and gives zeros."""
    V, D, ld, dt = _float_rows(table, "table")
    if not isinstance(ids, torch.Tensor) or ids.dim() != 1:
        raise TypeError("ids must be a 1-D int32 tensor")
    T, dev, given = ids.shape[0], table.device, out
    _vector(ids, T, dev, "ids", (torch.int32,))
    out, ldo = _float_out(out, T, D, table.dtype, dev, "out")
    _require_cuda(table, "table")
    _call(reqat_embedding, dev, ids.data_ptr(), T, table.data_ptr(), dt, V, D, ld, scale, out.data_ptr(), ldo)
    if given is not None:
        _written(given)
    return out


def embedding_backward(dy, ids, rows, scale=1.0, out=None, accumulate=False, out_dtype=None, ws=None):
    """Gradient of the table [rows, D] of embedding() from dy [T, D]: every id's rows of dy summed in float32, in a fixed
    order, times scale.  With accumulate it is added to ``out``, whose other rows stay untouched (a table that has a
    gradient already, as one that is the output layer's too).  out_dtype: default dy's, or out's.  ws: uint8 tensor of at
    least reqat_embedding_workspace_bytes(T, rows, D) bytes."""
    T, D, lddy, dt = _float_rows(dy, "dy")
    dev = dy.device
    _vector(ids, T, dev, "ids", (torch.int32,))
    if out is None and accumulate:
        raise ValueError("accumulate needs out")
    if out_dtype is None:
        out_dtype = dy.dtype if out is None else out.dtype
    out_dt, given = _dtype_arg(out_dtype), out
    out, ld = _float_out(out, rows, D, out_dtype, dev, "out")
    need = _embedding_workspace(T, rows, D)
    if ws is not None:
        _workspace_arg(ws, need, dev)
    _require_cuda(dy, "dy")
    if ws is None and need > 0:
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
    _call(reqat_embedding_backward, dev, dy.data_ptr(), dt, lddy, ids.data_ptr(), T, rows, D, scale, out.data_ptr(), out_dt,
          ld, 1 if accumulate else 0, _ptr(ws))
    if given is not None:
        _written(given)
    return out


_TENSORS = {torch.Tensor, torch.nn.Parameter}
_SHAPE, _DTYPE, _DEVICE = map(operator.attrgetter, ("shape", "dtype", "device"))


def _same_objects(a, b):
    return len(a) == len(b) and all(map(operator.is_, a, b))


class AdamW:
    """AdamW over many tensors in few launches, with states in 32 or 8 bits.

    params: contiguous tensors of one type, bfloat16 or float32, on one device, updated in place; copies: for each of them
    a bfloat16 tensor of the same shape that receives the new values rounded (the weights that the quantizers read, beside
    float32 master weights), or None.  The states of all tensors lie in one buffer each: ``m`` and ``v``, float32, or uint8
    codes with the float32 scales ``m_scale`` and ``v_scale`` of every 128 elements (the formats are stated in
    include/reqat.h); tensor i has the elements ``offsets[i]`` .. ``offsets[i]`` + its size.  All zeros at the start, they
    may be written in place or assigned.  ``steps`` counts the steps taken, ``missed[i]`` those of them that left parameter
    i out: its moments have moved steps - missed[i] times, and that count corrects their bias.  Both, ``lr``, ``betas``,
    ``eps`` and ``weight_decay`` may be assigned between steps.

    captured=True is for steps in a HIP graph: the count is ``step_tensor`` (int32) and the rate ``lr_tensor`` (float32),
    on the device, the count rising with every replay (``steps`` counts the steps outside of graphs).  It is one count for
    all: the first step says which parameters have gradients, and every later one has them for the same.  Parameters,
    copies, states and gradients of a captured step stay where they are."""

    def __init__(self, params, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, copies=None,
                 captured=False):
        self.params = list(params)
        self.copies = None if copies is None else list(copies)
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        if not self.params:
            raise ValueError("no parameters")
        first = self.params[0]
        if not isinstance(first, torch.Tensor) or first.dtype not in _FLOATS:
            raise TypeError("parameters must be bfloat16 or float32 tensors")
        self.device, self.dtype, self.state_bits = first.device, first.dtype, state_bits
        self._shapes = [p.shape if isinstance(p, torch.Tensor) else None for p in self.params]
        # an array of reqat_adamw_tensor; a step fills in the addresses of gradients, and what has changed
        self._tensors = array.array("q", bytes(64 * len(self.params)))
        self._adopt()
        self.lr, self.betas, self.eps, self.weight_decay, self.steps = lr, betas, eps, weight_decay, 0
        self.offsets, size = [], 0
        for p in self.params:
            self.offsets.append(size)
            size += -(-p.numel() // 128) * 128
        kind = torch.float32 if state_bits == 32 else torch.uint8
        self.m, self.v = (torch.zeros(size, dtype=kind, device=self.device) for _ in range(2))
        self.m_scale = self.v_scale = None
        if state_bits == 8:
            self.m_scale, self.v_scale = (torch.zeros(size // 128, dtype=torch.float32, device=self.device) for _ in range(2))
        self._sizes = array.array("q", [p.numel() for p in self.params])
        self._total, self._bases = size, None
        self.missed = [0] * len(self.params)
        self.step_tensor = self.lr_tensor = self._coef = self._stepped = None
        if captured:
            self.step_tensor = torch.zeros(1, dtype=torch.int32, device=self.device)
            self.lr_tensor = torch.full((1,), lr, dtype=torch.float32, device=self.device)
            self._coef = torch.zeros(3, dtype=torch.float32, device=self.device)

    def _tensors_now(self):
        return [*self.params, *(self.copies or ())]

    def _adopt(self):
        """Checks parameters and copies, enters their addresses and holds on to their memory, so that an address that stays
        is theirs."""
        spans, held = [], []
        if len(self.params) != len(self._shapes):
            raise ValueError("params must stay %d tensors" % len(self._shapes))
        if self.copies is not None and len(self.copies) != len(self.params):
            raise ValueError("copies must have one tensor (or None) for each parameter")
        for i, (p, shape) in enumerate(zip(self.params, self._shapes)):
            self._tensor_arg(p, shape, (self.dtype,), "params[%d]" % i)
            c = None if self.copies is None else self.copies[i]
            if c is not None:
                self._tensor_arg(c, shape, (torch.bfloat16,), "copies[%d]" % i)
            for t in (p, c):
                if t is not None and t.numel():
                    spans.append((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size()))
                    held.append(t.detach())
        spans.sort()
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("parameters and copies must not overlap")
        self._held, self._seen = held, self._tensors_now()
        self._live = [t for t in self._seen if t is not None]
        self._addresses = list(map(torch.Tensor.data_ptr, self._live))
        copies = self.copies if self.copies is not None else [None] * len(self.params)
        self._tensors[0::8] = array.array("q", [p.data_ptr() for p in self.params])
        self._tensors[6::8] = array.array("q", [0 if c is None else c.data_ptr() for c in copies])

    def _place_states(self, bases):
        """Checks the states' buffers and enters their addresses: at the first step, and when one was replaced."""
        kind = torch.float32 if self.state_bits == 32 else torch.uint8
        for name, n, dtype in (("m", self._total, kind), ("v", self._total, kind),
                               ("m_scale", self._total // 128, torch.float32), ("v_scale", self._total // 128, torch.float32)):
            if dtype is torch.float32 and self.state_bits == 32 and name.endswith("scale"):
                continue
            _index_arg(getattr(self, name), (n,), dtype, self.device, name)
        spans = sorted((t.data_ptr(), t.data_ptr() + t.numel() * t.element_size())
                       for t in (self.m, self.v, self.m_scale, self.v_scale) if t is not None and t.numel())
        if any(a[1] > b[0] for a, b in zip(spans, spans[1:])):
            raise ValueError("the states' buffers must not overlap")
        for i, at in enumerate(self.offsets):
            self._tensors[8 * i + 2] = bases[0] + at * self.m.element_size()
            self._tensors[8 * i + 3] = bases[1] + at * self.v.element_size()
            if self.state_bits == 8:
                self._tensors[8 * i + 4] = bases[2] + at // 32
                self._tensors[8 * i + 5] = bases[3] + at // 32
        self._bases, self._seen_states = bases, [self.m, self.v, self.m_scale, self.v_scale]
        self._held_states = [t if t is None else t.detach() for t in (self.m, self.v, self.m_scale, self.v_scale)]

    def _tensor_arg(self, t, shape, dtypes, name):
        if not isinstance(t, torch.Tensor) or t.dtype not in dtypes:
            raise TypeError("%s must be a tensor of %s" % (name, " or ".join(str(d) for d in dtypes)))
        if t.shape != shape:
            raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
        if not t.is_contiguous():
            raise ValueError("%s must be contiguous" % name)
        _same_device(t, self.device, name)

    def _all_as_expected(self, grads, kind):
        """Whether every gradient is a tensor of its parameter's shape: the checks of many small tensors, one attribute at a
        time."""
        return (kind in _FLOATS and set(map(type, grads)) <= _TENSORS and list(map(_SHAPE, grads)) == self._shapes
                and set(map(_DTYPE, grads)) == {kind} and set(map(_DEVICE, grads)) == {self.device}
                and all(map(torch.Tensor.is_contiguous, grads)))

    def step(self, grads, grad_scale=None):
        """One step with the gradients of all parameters (tensors of their shapes, all bfloat16 or all float32; None: the
        parameter is left out of this step, its count too), each times grad_scale (a float32 tensor of one element, as
        of a clipped norm) first.  Parameters of different counts go in launches of their own."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("grads must have one tensor (or None) for each parameter")
        if grad_scale is not None:
            _scale_arg(grad_scale, NVFP4, self.device, "grad_scale")
        kind = next((g.dtype for g in grads if isinstance(g, torch.Tensor)), torch.float32)
        sizes, dev = self._sizes, self.device
        if self._all_as_expected(grads, kind):
            at = list(map(torch.Tensor.data_ptr, grads))
        else:
            at, sizes = [], sizes[:]
            for i, (g, shape) in enumerate(zip(grads, self._shapes)):
                if g is None:
                    sizes[i] = 0                         # left out
                else:
                    self._tensor_arg(g, shape, (kind,) if kind in _FLOATS else tuple(_FLOATS), "grads[%d]" % i)
                at.append(0 if g is None else g.data_ptr())
        # another tensor, perhaps in the same memory, or one that was given other memory
        if not _same_objects(self._tensors_now(), self._seen) or list(map(torch.Tensor.data_ptr, self._live)) != self._addresses:
            self._adopt()
        states = [self.m, self.v, self.m_scale, self.v_scale]
        bases = [0 if t is None else t.data_ptr() for t in states]
        if bases != self._bases or not _same_objects(states, self._seen_states):
            self._place_states(bases)
        tensors, count = self._tensors, len(at)
        tensors[1::8] = array.array("q", at)
        _require_cuda(self.params[0], "params[0]")
        if self._coef is not None:
            self._step_captured(grads, kind, sizes, grad_scale)
            self._step_written(grads)
            return
        missed = self.missed
        if not any(missed):
            behind = (0,)
        else:                                            # the lowest count first: it is the one that may be refused
            behind = sorted({n for n, size in zip(missed, sizes) if size}, reverse=True)
        for n in behind:
            tensors[7::8] = sizes if len(behind) == 1 else array.array("q", [z if k == n else 0 for z, k in zip(sizes, missed)])
            _call(reqat_adamw_step, dev, tensors, count, _FLOATS[self.dtype], _FLOATS[kind], self.state_bits,
                  self._hyper(self.steps + 1 - n), _ptr(grad_scale), None)
        if sizes is not self._sizes:
            self.missed = [k + (g is None) for k, g in zip(missed, grads)]
        self.steps += 1
        self._step_written(grads)

    def _step_written(self, grads):
        written = self._live
        if any(g is None for g in grads):
            written = [t for t, g in zip(self._seen, [*grads, *grads]) if t is not None and g is not None]
        _written(*written)

    def _hyper(self, step):
        return AdamwHyper(self.lr, *self.betas, self.eps, self.weight_decay, step)

    def _step_captured(self, grads, kind, sizes, grad_scale):
        stepped = [g is not None for g in grads]
        if self._stepped is None and not any(stepped):
            return
        if self._stepped not in (None, stepped):
            raise ValueError("captured steps have gradients for the same parameters each time")
        hyper = self._hyper(1)                           # the count is on the device
        self._tensors[7::8] = sizes
        _call(reqat_adamw_coefficients, self.device, hyper, self.lr_tensor.data_ptr(), self.step_tensor.data_ptr(),
              self._coef.data_ptr())
        _call(reqat_adamw_step, self.device, self._tensors, len(grads), _FLOATS[self.dtype], _FLOATS[kind], self.state_bits,
              hyper, _ptr(grad_scale), _ptr(self._coef))
        self._stepped = stepped
        with torch.cuda.device(self.device):
            if not torch.cuda.is_current_stream_capturing():
                self.steps += 1

    def moments(self):
        """The values of m and v as float32 buffers laid out like them (the states themselves when they have 32 bits)."""
        if self.state_bits == 32:
            return self.m, self.v
        _require_cuda(self.m, "m")
        n = self._total
        for name, shape, dtype in (("m", (n,), torch.uint8), ("v", (n,), torch.uint8), ("m_scale", (n // 128,), torch.float32),
                                   ("v_scale", (n // 128,), torch.float32)):
            _index_arg(getattr(self, name), shape, dtype, self.device, name)
        m, v = (torch.empty(n, dtype=torch.float32, device=self.device) for _ in range(2))
        _call(reqat_adamw_moments, self.device, self.m.data_ptr(), self.m_scale.data_ptr(), self.v.data_ptr(),
              self.v_scale.data_ptr(), n, m.data_ptr(), v.data_ptr())
        return m, v


class PolicyLoss(torch.autograd.Function):
    """The policy loss as an autograd function over the logits; the arguments of policy_loss() in order."""

    @staticmethod
    def forward(ctx, logits, targets, old_logp, advantages, ref_logp=None, weights=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0, temperature=1.0):
        loss, stats = policy_loss(logits, targets, old_logp, advantages, ref_logp, weights, clip_low, clip_high, kl_coef,
                                  temperature)
        ctx.save_for_backward(logits, targets, stats)
        ctx.temperature = temperature
        return loss[0]

    @staticmethod
    def backward(ctx, g):
        logits, targets, stats = ctx.saved_tensors
        grad = policy_loss_backward(logits, targets, stats, ctx.temperature, g.reshape(1).to(torch.float32))
        return _once("PolicyLoss", (grad,), g, logits) + (None,) * 9


class LayerNorm(torch.autograd.Function):
    """layer_norm() as an autograd function of x, weight and bias."""

    @staticmethod
    def forward(ctx, x, weight, bias=None, eps=1e-6, center=True):
        y, stats = layer_norm(x, weight, bias, eps, center)
        ctx.save_for_backward(x, weight, stats)
        ctx.center, ctx.bias = center, bias is not None
        return y

    @staticmethod
    def backward(ctx, dy):
        x, weight, stats = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(_dense_rows(dy), x, weight, stats, ctx.center, ctx.bias)
        return _once("LayerNorm", (dx, dw, db), dy, x, weight) + (None, None)


class Embedding(torch.autograd.Function):
    """embedding() as an autograd function of the table (ids come first, as in embedding())."""

    @staticmethod
    def forward(ctx, ids, table, scale=1.0):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.scale = table.shape[0], scale
        return embedding(ids, table, scale)

    @staticmethod
    def backward(ctx, dy):
        ids, = ctx.saved_tensors
        dtable = embedding_backward(_dense_rows(dy), ids, ctx.rows, ctx.scale)
        return (None,) + _once("Embedding", (dtable,), dy) + (None,)


def _dense_rows(g):
    """A gradient as the kernels take it: one that autograd expanded has rows without an extent of their own."""
    return g if g.stride(1) == 1 and g.stride(0) >= g.shape[1] else g.contiguous()
