"""ctypes binding of libdard.so (include/dard.h).

Every function here only marshals arguments: torch tensors become device
pointers, shapes become sizes, the current torch stream becomes the HIP
stream.  All computation happens in the HIP kernels of libdard.so; if the
library is missing, loading fails loudly -- there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdard.so")

DARD_OK = 0
STATE_M, STATE_C, STATE_U = 0, 1, 2
DTYPE_F32, DTYPE_BF16, DTYPE_BF16_KV_FP8 = 0, 1, 2
KV_DTYPE, KV_FP8 = 0, 1
MX_FP8, MX_FP4 = 0, 1
MX_BLOCK = 32
F_XSELF_SHADOW, F_MKEYS_SHADOW, F_VERIFY_PCUR, F_PROGRESS = 1, 2, 4, 8
F_C_BIDIR, F_ORDER_L2R, F_ORDER_ENTROPY, F_ORDER_MARGIN, F_FIXED_W = 16, 32, 64, 128, 256
F_CHECK_STATES = 512
F_HIDDEN_MIX = 1024
BAD_STATE = -1
GEMM_STREAM, GEMM_PIPE, GEMM_BIG, GEMM_TILED, GEMM_F32 = range(5)
PHASE_VERIFY, PHASE_FINAL = 0, 1
(K_GEMM_QKV, K_GEMM_O, K_GEMM_GU, K_GEMM_DOWN, K_GEMM_HEAD, K_ATTENTION, K_CONFIDENCE,
 K_DECIDE, K_NORM, K_MASK, K_COUNT) = range(11)

EXPORTS = [
    "dard_last_error", "dard_version", "dard_check_states", "dard_build_state_mask", "dard_attention_workspace_bytes",
    "dard_masked_attention", "dard_confidence_workspace_bytes", "dard_confidence", "dard_confidence_noalloc",
    "dard_commit_remask", "dard_packed_weight_bytes", "dard_pack_weights", "dard_kv_bytes",
    "dard_workspace_bytes", "dard_prefill", "dard_prefill_extend", "dard_step", "dard_step_full", "dard_prefill_suffix",
    "dard_step_shared", "dard_pack_matrix", "dard_linear", "dard_gemm_plan",
    "dard_quantize_mx", "dard_dequantize_mx", "dard_resid_norm_mx", "dard_packed_mx_bytes", "dard_pack_matrix_mx",
    "dard_linear_mx_workspace_bytes", "dard_linear_mx", "dard_linear_mx_plan", "dard_kv_write_mx", "dard_kv_read_mx",
    "dard_attention_mx_workspace_bytes", "dard_masked_attention_mx",
    "dard_attention_shared_workspace_bytes", "dard_masked_attention_shared", "dard_key_weights_workspace_bytes",
    "dard_key_weights", "dard_kv_select_workspace_bytes", "dard_kv_select", "dard_kv_compact",
    "dard_trace_enable",
    "dard_trace_read", "dard_trace_reset", "dard_trace_sample",
]


class DardError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"libdard status {status}: {msg}")
        self.status = status


class dard_params(ctypes.Structure):
    _fields_ = [("tau_c", ctypes.c_float), ("tau_u", ctypes.c_float), ("lambda_", ctypes.c_double),
                ("p0", ctypes.c_double), ("mask_id", ctypes.c_int32), ("flags", ctypes.c_uint32),
                ("w_fixed", ctypes.c_float)]


class dard_dims(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "head_dim",
                                              "ffn_dim", "vocab", "max_pos", "dtype")] + \
               [("norm_eps", ctypes.c_float), ("rope_theta", ctypes.c_float), ("kv_format", ctypes.c_int32)]


class dard_step_debug(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("logits", "w", "maxprob_s", "argmax_s", "pcur_s",
                                               "maxprob_mix", "argmax_mix", "entropy", "margin")]


_lib = None


def lib():
    """Load libdard.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, u32, sz, f32, i64 = (ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32, ctypes.c_size_t,
                                      ctypes.c_float, ctypes.c_int64)
        sig = {
            "dard_last_error": (ctypes.c_char_p, []),
            "dard_version": (i32, []),
            "dard_check_states": (i32, [vp, i32, vp, vp]),
            "dard_build_state_mask": (i32, [vp, vp, i32, i32, u32, vp, vp]),
            "dard_attention_workspace_bytes": (sz, [i32, i32, i32, i32, i32, i32]),
            "dard_masked_attention": (i32, [i32, vp, vp, vp, i32, i32, vp, vp, i32, i32, i32, i32, i32, f32,
                                            u32, vp, vp, sz, vp]),
            "dard_confidence_workspace_bytes": (sz, [i32, i32]),
            "dard_confidence": (i32, [vp, vp, vp, vp, i32, i32, i64, vp, vp, vp, vp, vp, vp, sz, vp]),
            "dard_confidence_noalloc": (i32, [vp, vp, vp, vp, i32, i32, i64, vp, vp, vp, vp, vp, vp]),
            "dard_commit_remask": (i32, [i32, vp, i32, i32] + [vp] * 14),
            "dard_packed_weight_bytes": (sz, [vp]),
            "dard_pack_weights": (i32, [vp, vp, i32, vp, sz, vp]),
            "dard_kv_bytes": (sz, [vp, i32, i32]),
            "dard_workspace_bytes": (sz, [vp, i32, i32, i32]),
            "dard_prefill": (i32, [vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]),
            "dard_step": (i32, [vp, vp, vp, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            "dard_step_full": (i32, [vp, vp, vp, i32, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz,
                                     vp]),
            "dard_prefill_suffix": (i32, [vp, vp, vp, i32, vp, i32, i32, i32, i32, vp, vp, sz, vp]),
            "dard_prefill_extend": (i32, [vp, vp, vp, i32, i32, i32, i32, vp, vp, sz, vp]),
            "dard_step_shared": (i32, [vp, vp, vp, i32, vp, i32, i32, i32, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp,
                                       vp, vp, sz, vp]),
            "dard_pack_matrix": (i32, [i32, vp, i32, i32, vp, vp]),
            "dard_linear": (i32, [i32, vp, i32, i32, vp, i32, vp, vp]),
            "dard_gemm_plan": (i32, [i32, i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_int32)]),
            "dard_quantize_mx": (i32, [i32, vp, i64, i32, i32, i32, vp, vp, vp]),
            "dard_dequantize_mx": (i32, [i32, vp, vp, i32, i32, i32, vp, i64, vp]),
            "dard_resid_norm_mx": (i32, [vp, i32, vp, i32, vp, f32, i32, i32, i32, vp, vp, vp]),
            "dard_packed_mx_bytes": (sz, [i32, i32]),
            "dard_pack_matrix_mx": (i32, [vp, vp, i32, i32, vp, vp]),
            "dard_linear_mx_workspace_bytes": (sz, [i32, i32, i32, i32]),
            "dard_linear_mx": (i32, [i32, vp, vp, i32, i32, vp, i32, i32, vp, vp, sz, vp]),
            "dard_linear_mx_plan": (i32, [i32, i32, i32, i32, i32, ctypes.POINTER(ctypes.c_int32)]),
            "dard_kv_write_mx": (i32, [i32, vp, vp, i64, i32, i32, i32, i32, i32, vp, i32, vp, vp, vp, vp, vp]),
            "dard_kv_read_mx": (i32, [vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, vp, i32, vp, vp, i64, vp]),
            "dard_attention_mx_workspace_bytes": (sz, [i32, i32, i32, i32, i32, i32]),
            "dard_masked_attention_mx": (i32, [vp, vp, vp, vp, vp, i32, vp, i32, vp, vp, i32, i32, i32, i32, i32, f32,
                                               u32, vp, vp, sz, vp]),
            "dard_attention_shared_workspace_bytes": (sz, [i32] * 8),
            "dard_masked_attention_shared": (i32, [i32, vp, vp, vp, i32, i32, vp, vp, i32, vp, i32, vp, vp, i32, i32, i32,
                                                   i32, i32, f32, u32, vp, vp, vp, sz, vp]),
            "dard_key_weights_workspace_bytes": (sz, [i32] * 7),
            "dard_key_weights": (i32, [i32, vp, vp, vp, i32, vp, i32, i32, i32, i32, i32, i32, f32, f32, vp, i64, vp, sz,
                                       vp]),
            "dard_kv_select_workspace_bytes": (sz, [i32] * 4),
            "dard_kv_select": (i32, [vp, i64, i32, vp, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]),
            "dard_kv_compact": (i32, [i32, vp, vp, i32, vp, i64, vp, i32, vp, i32, vp, i32, i32, i32, vp]),
            "dard_trace_enable": (i32, [u32]),
            "dard_trace_read": (i32, [i32, ctypes.POINTER(i64), ctypes.POINTER(ctypes.c_double)]),
            "dard_trace_reset": (i32, []),
            "dard_trace_sample": (i32, [i32]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status):
    if status != DARD_OK:
        raise DardError(status, lib().dard_last_error().decode())
    return status


def _p(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        return t
    if not t.is_cuda:
        raise ValueError("libdard takes device tensors")
    if not t.is_contiguous():
        raise ValueError("libdard takes contiguous tensors")
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else stream


def _dt(t):
    return DTYPE_BF16 if t.dtype == torch.bfloat16 else DTYPE_F32


def _ref(x):
    return ctypes.byref(x) if x is not None else None


def make_params(tau_c=0.4, tau_u=0.9, lam=0.5 ** (1 / 8), p0=0.1, mask_id=0, flags=0, w_fixed=0.0):
    return dard_params(tau_c, tau_u, lam, p0, mask_id, flags, w_fixed)


def make_dims(d):
    """From a synth.Dims (or anything with the same attributes)."""
    kv = getattr(d, "kv_dtype", "")
    if kv not in ("", "fp8", d.dtype):
        raise ValueError(f"unknown kv_dtype {kv!r}")
    return dard_dims(d.n_layers, d.d_model, d.n_heads, d.n_kv_heads, d.head_dim, d.ffn_dim, d.vocab, d.max_pos,
                     DTYPE_BF16 if d.dtype == "bf16" else DTYPE_F32, d.norm_eps, d.rope_theta,
                     KV_FP8 if kv == "fp8" else KV_DTYPE)


# ------------------------------------------------------------------ entry points
def dard_version():
    return lib().dard_version()


def dard_check_states(state, status, stream=None):
    """status (int32 [2] on the device) = (codes outside {0,1,2}, first index or -1)."""
    _check(lib().dard_check_states(_p(state), state.numel(), _p(status), _stream(stream)))


def dard_gemm_plan(M, N, K, partial=False, frag_x=True, dtype=DTYPE_BF16):
    """(kernel, tile rows / 32, tile columns / 32, K split) the library runs for
    a projection of these sizes."""
    plan = (ctypes.c_int32 * 4)()
    _check(lib().dard_gemm_plan(dtype, M, N, K, int(partial), int(frag_x), plan))
    return tuple(plan)


def dard_build_state_mask(state, conf, flags, sel, stream=None):
    b, B = state.shape
    _check(lib().dard_build_state_mask(_p(state), _p(conf), b, B, flags, _p(sel), _stream(stream)))


def dard_attention_workspace_bytes(dtype, b, B, Hq, dh, P):
    return lib().dard_attention_workspace_bytes(dtype, b, B, Hq, dh, P)


def dard_masked_attention(q, k, v, P, state, conf, scale, flags, out, ws=None, stream=None):
    """q [b][2B][Hq][dh], k [b][Hkv][cap][dh], v [b][Hkv][dh][cap] (dims-major);
    uint8 k / v hold OCP FP8 E4M3 codes (bf16 q / out)."""
    b, R, Hq, dh = q.shape
    _, Hkv, cap, _ = k.shape
    if tuple(v.shape) != (b, Hkv, dh, cap):
        raise ValueError(f"v must be [b][Hkv][dh][cap] = {(b, Hkv, dh, cap)}, got {tuple(v.shape)}")
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    dt = DTYPE_BF16_KV_FP8 if k.dtype == torch.uint8 else _dt(q)
    _check(lib().dard_masked_attention(dt, _p(q), _p(k), _p(v), P, cap, _p(state), _p(conf), b, R // 2, Hq,
                                       Hkv, dh, scale, flags, _p(out), _p(ws), nbytes, _stream(stream)))


def dard_confidence_workspace_bytes(rows, V):
    return lib().dard_confidence_workspace_bytes(rows, V)


def dard_confidence(logits_s, argmax, maxprob, logits_x=None, w=None, cur_tok=None, pcur=None, ws=None,
                    stream=None, entropy=None, margin=None):
    rows, V = logits_s.shape
    nbytes = ws.numel() * ws.element_size() if ws is not None else 0
    _check(lib().dard_confidence(_p(logits_s), _p(logits_x), _p(w), _p(cur_tok), rows, V, logits_s.stride(0),
                                 _p(argmax), _p(maxprob), _p(pcur), _p(entropy), _p(margin), _p(ws), nbytes,
                                 _stream(stream)))


def dard_confidence_noalloc(logits_s, argmax, maxprob, logits_x=None, w=None, cur_tok=None, pcur=None,
                            stream=None, entropy=None, margin=None):
    """dard_confidence with the library's preallocated scratch (no workspace)."""
    rows, V = logits_s.shape
    _check(lib().dard_confidence_noalloc(_p(logits_s), _p(logits_x), _p(w), _p(cur_tok), rows, V,
                                         logits_s.stride(0), _p(argmax), _p(maxprob), _p(pcur), _p(entropy),
                                         _p(margin), _stream(stream)))


def dard_commit_remask(phase, params, state_in, maxprob_s=None, pcur_s=None, argmax_s=None, maxprob_mix=None,
                       argmax_mix=None, w_out=None, state_out=None, tok_out=None, conf_out=None,
                       block_done=None, stream=None, key_s=None, key_mix=None):
    b, B = state_in.shape
    _check(lib().dard_commit_remask(phase, ctypes.byref(params), b, B, _p(state_in), _p(maxprob_s), _p(pcur_s),
                                    _p(argmax_s), _p(maxprob_mix), _p(argmax_mix), _p(key_s), _p(key_mix),
                                    _p(w_out), _p(state_out), _p(tok_out), _p(conf_out), _p(block_done),
                                    _stream(stream)))


def dard_pack_matrix(W, Wp, stream=None):
    N, K = W.shape
    _check(lib().dard_pack_matrix(_dt(W), _p(W), N, K, _p(Wp), _stream(stream)))


def dard_linear(X, Wp, N, Y, stream=None):
    """Y = X W^T with W packed by dard_pack_matrix (Wp has N*K elements)."""
    M, K = X.shape
    _check(lib().dard_linear(_dt(X), _p(X), M, K, _p(Wp), N, _p(Y), _stream(stream)))


def _mx_check(rows, K, format, codes, scales):
    """codes and scales of `rows` rows of K values."""
    if format != MX_FP8 and format != MX_FP4:
        raise ValueError(f"unknown MX format {format!r}")
    if K % MX_BLOCK:
        raise ValueError(f"MX rows hold whole blocks of {MX_BLOCK} values, got {K}")
    if codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8:
        raise ValueError("MX codes and scales are uint8 tensors")
    want = rows * (K if format == MX_FP8 else K // 2)
    if codes.numel() != want or scales.numel() != rows * (K // MX_BLOCK):
        raise ValueError(f"need {want} code bytes and {rows * (K // MX_BLOCK)} scales for {rows} rows of {K}, got "
                         f"{codes.numel()} and {scales.numel()}")


def _mx_dt(t, what):
    if t.dtype is torch.bfloat16:
        return DTYPE_BF16
    if t.dtype is torch.float32:
        return DTYPE_F32
    raise ValueError(f"{what} must be bfloat16 or float32, got {t.dtype}")


def _args(stream, tensors, strided=()):
    """Device pointers of contiguous tensors (None -> NULL), then of `strided` ones, and the HIP stream
    of the call.  All must be on the current device: kernels launch there."""
    dev = torch._C._cuda_getDevice() if torch.cuda.is_initialized() else -1
    ptrs = []
    for t in tensors:
        if t is None:
            ptrs.append(None)
            continue
        d = t.get_device()
        if d != dev or d < 0:
            _wrong_device(d, dev)
        if not t.is_contiguous():
            raise ValueError("libdard takes contiguous tensors")
        ptrs.append(t.data_ptr())
    for t in strided:
        d = t.get_device()
        if d != dev or d < 0:
            _wrong_device(d, dev)
        ptrs.append(t.data_ptr())
    if stream is None:
        return ptrs, torch._C._cuda_getCurrentRawStream(dev)
    return ptrs, _stream(stream)


def _wrong_device(d, dev):
    if d < 0:
        raise ValueError("libdard takes device tensors")
    raise ValueError(f"tensor on cuda:{d}, but the current device is cuda:{dev}")


def _rows_ld(t, what):
    """Leading dimension of a [rows][K] tensor whose rows are contiguous."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be [rows][K] with contiguous rows")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _nbytes(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


def dard_quantize_mx(x, format, codes, scales, stream=None):
    """x [rows][K] (bf16 or float32, rows may be further apart) to MX codes
    (uint8 [rows][K] or, MX_FP4, [rows][K/2]) and scales (uint8 [rows][K/32])."""
    ld = _rows_ld(x, "x")
    rows, K = x.shape
    _mx_check(rows, K, format, codes, scales)
    dt = _mx_dt(x, "x")
    (c, s, p), st = _args(stream, (codes, scales), (x,))
    _check(lib().dard_quantize_mx(dt, p, ld, rows, K, format, c, s, st))


def dard_dequantize_mx(format, codes, scales, x, stream=None):
    """The values of MX codes and scales into x [rows][K] (bf16 or float32)."""
    ld = _rows_ld(x, "x")
    rows, K = x.shape
    _mx_check(rows, K, format, codes, scales)
    dt = _mx_dt(x, "x")
    (c, s, p), st = _args(stream, (codes, scales), (x,))
    _check(lib().dard_dequantize_mx(format, c, s, rows, K, dt, p, ld, st))


def dard_resid_norm_mx(h, gain, eps, format, codes, scales, delta=None, stream=None):
    """h [rows][d] float32 += delta (bf16 or float32, or None); the RMS norm of
    its rows times gain in MX."""
    rows, d = h.shape
    if h.dtype is not torch.float32:
        raise ValueError("h must be float32")
    if gain.numel() != d or (delta is not None and delta.shape != h.shape):
        raise ValueError(f"need gain [{d}] and delta [{rows}][{d}]")
    _mx_check(rows, d, format, codes, scales)
    ddt, gdt = DTYPE_F32 if delta is None else _mx_dt(delta, "delta"), _mx_dt(gain, "gain")
    (hp, dp, gp, c, s), st = _args(stream, (h, delta, gain, codes, scales))
    _check(lib().dard_resid_norm_mx(hp, ddt, dp, gdt, gp, eps, rows, d, format, c, s, st))


def dard_packed_mx_bytes(N, K):
    n = lib().dard_packed_mx_bytes(N, K)
    if n == 0:
        raise DardError(-2, lib().dard_last_error().decode())
    return n


def dard_pack_matrix_mx(codes, scales, Wp, stream=None):
    """Lay out MXFP4 weights (codes [N][K/2], scales [N][K/32]) for dard_linear_mx;
    Wp: uint8 [dard_packed_mx_bytes(N, K)]."""
    N, K = codes.shape[0], 2 * codes.shape[1]
    _mx_check(N, K, MX_FP4, codes, scales)
    if _nbytes(Wp) < dard_packed_mx_bytes(N, K):
        raise ValueError(f"Wp needs {dard_packed_mx_bytes(N, K)} bytes")
    (c, s, w), st = _args(stream, (codes, scales, Wp))
    _check(lib().dard_pack_matrix_mx(c, s, N, K, w, st))


def dard_linear_mx_workspace_bytes(format, M, N, K):
    return lib().dard_linear_mx_workspace_bytes(format, M, N, K)


def dard_linear_mx_plan(format, M, N, K, out=torch.float32):
    """(workgroup rows, workgroup columns, parts of K in a workgroup or 0, exact products) that the library runs
    for a product with results of type `out`."""
    if out is not torch.float32 and out is not torch.bfloat16:
        raise ValueError(f"out must be bfloat16 or float32, got {out}")
    plan = (ctypes.c_int32 * 4)()
    _check(lib().dard_linear_mx_plan(format, M, N, K, DTYPE_BF16 if out is torch.bfloat16 else DTYPE_F32, plan))
    return tuple(plan)


def dard_linear_mx(format, codes, scales, Wp, Y, ws=None, stream=None):
    """Y [M][N] (bf16 or float32) = X W^T, X in MX (codes [M][K] or [M][K/2],
    scales [M][K/32]), W packed by dard_pack_matrix_mx."""
    M, N = Y.shape
    K = codes.shape[1] * (1 if format == MX_FP8 else 2)
    _mx_check(M, K, format, codes, scales)
    if _nbytes(Wp) < -(-N // 32) * -(-K // 256) * 4352:   # (dard_packed_mx_bytes: 32 x 256 values a block, 17 bytes for 32)
        raise ValueError(f"Wp of {_nbytes(Wp)} bytes does not hold a packed [{N}][{K}] matrix")
    dt = _mx_dt(Y, "Y")
    (c, s, w, y, room), st = _args(stream, (codes, scales, Wp, Y, ws))
    _check(lib().dard_linear_mx(format, c, s, M, K, w, N, dt, y, room, _nbytes(ws), st))


def _mx_cache(cache, b, Hkv, dh):
    """Capacity of an MXFP4 cache (kc, ks, vc, vs) of b sequences."""
    kc, ks, vc, vs = cache
    shape = kc.shape
    if len(shape) != 4:
        raise ValueError("kc must be [b][Hkv][cap][dh/2]")
    cap, u8 = shape[2], torch.uint8
    want = ((b, Hkv, cap, dh // 2), (b, Hkv, cap, dh // 32), (b, Hkv, cap // 8, dh // 4, 8, 2),
            (b, Hkv, cap // 8, dh // 32, 8))
    if not (shape == want[0] and ks.shape == want[1] and vc.shape == want[2] and vs.shape == want[3] and kc.dtype is u8
            and ks.dtype is u8 and vc.dtype is u8 and vs.dtype is u8):
        for name, t, w in zip(("kc", "ks", "vc", "vs"), cache, want):
            if t.shape != w or t.dtype is not u8:
                raise ValueError(f"{name} must be uint8 {w}, got {t.dtype} {tuple(t.shape)}")
    return cap


def _mx_prefix(prefix, b):
    if prefix is not None and (prefix.dtype is not torch.int32 or prefix.numel() != b):
        raise ValueError(f"prefix must be int32 [{b}]")
    return prefix


def _tokens_ld(shape, stride, what):
    """Elements between the tokens of a [b][n][Hkv][dh] tensor whose heads are contiguous."""
    b, n, Hkv, dh = shape
    sb, sn, sh, sd = stride
    ld = sn if n > 1 else (sb if b > 1 else Hkv * dh)
    if (dh > 1 and sd != 1) or (Hkv > 1 and sh != dh) or (b > 1 and sb != n * ld):
        raise ValueError(f"{what} must be [b][n][Hkv][dh] with contiguous heads and evenly spaced tokens")
    return ld


def _kv_args(cache, k, v, prefix, stream):
    shape = k.shape
    if v.shape != shape or k.dtype is not v.dtype or len(shape) != 4:
        raise ValueError("k and v must be [b][n][Hkv][dh] tensors of one type")
    b, n, Hkv, dh = shape
    cap = _mx_cache(cache, b, Hkv, dh)
    stride, other = k.stride(), v.stride()
    ld = _tokens_ld(shape, stride, "k")
    if other != stride and _tokens_ld(shape, other, "v") != ld:
        raise ValueError("k and v must have the same distance between tokens")
    dt = _mx_dt(k, "k")
    ptrs, st = _args(stream, (*cache, _mx_prefix(prefix, b)), (k, v))
    return b, n, Hkv, dh, cap, ld, dt, ptrs, st


def dard_kv_write_mx(k, v, cache, pos, prefix=None, stream=None):
    """k, v [b][n][Hkv][dh] (bf16 or float32; slices of a wider row will do) into
    the MXFP4 cache (kc, ks, vc, vs) at keys pos.. (or prefix[s]..)."""
    b, n, Hkv, dh, cap, ld, dt, (kc, ks, vc, vs, pre, kp, vp), st = _kv_args(cache, k, v, prefix, stream)
    _check(lib().dard_kv_write_mx(dt, kp, vp, ld, b, n, Hkv, dh, pos, pre, cap, kc, ks, vc, vs, st))


def dard_kv_read_mx(cache, pos, k, v, prefix=None, stream=None):
    """The values of keys pos.. (or prefix[s]..) of the cache into k, v [b][n][Hkv][dh]."""
    b, n, Hkv, dh, cap, ld, dt, (kc, ks, vc, vs, pre, kp, vp), st = _kv_args(cache, k, v, prefix, stream)
    _check(lib().dard_kv_read_mx(kc, ks, vc, vs, cap, b, n, Hkv, dh, pos, pre, dt, kp, vp, ld, st))


def dard_attention_mx_workspace_bytes(b, B, Hq, Hkv, dh, P):
    return lib().dard_attention_mx_workspace_bytes(b, B, Hq, Hkv, dh, P)


def dard_masked_attention_mx(q, cache, P, state, conf, scale, flags, out, ws=None, prefix=None, stream=None):
    """dard_masked_attention over an MXFP4 cache (kc, ks, vc, vs); prefix: int32
    [b] prefix lengths of the sequences (at most P), or None: P each."""
    b, R, Hq, dh = q.shape
    if q.dtype is not torch.bfloat16 or out.dtype is not torch.bfloat16 or out.shape != q.shape:
        raise ValueError("q and out must be bfloat16 [b][2B][Hq][dh]")
    if R % 2 or state.shape != (b, R // 2) or conf.shape != state.shape:
        raise ValueError(f"state and conf must be [b][B] = {(b, R // 2)}")
    if state.dtype is not torch.uint8 or conf.dtype is not torch.float32:
        raise ValueError("state must be uint8, conf float32")
    Hkv = cache[0].shape[1]
    cap = _mx_cache(cache, b, Hkv, dh)
    (qp, kc, ks, vc, vs, pre, sp, cp, op, room), st = _args(stream, (q, *cache, _mx_prefix(prefix, b), state, conf, out, ws))
    _check(lib().dard_masked_attention_mx(qp, kc, ks, vc, vs, P, pre, cap, sp, cp, b, R // 2, Hq, Hkv, dh, scale, flags,
                                          op, room, _nbytes(ws), st))


def _kv_dt(q, *caches):
    """Operation type of q (or None) and the caches; FP8 caches hold E4M3 codes as uint8 or float8_e4m3fn."""
    kt = caches[0].dtype
    for t in caches:
        if t is not None and t.dtype is not kt:
            raise ValueError(f"the caches must have one type, got {kt} and {t.dtype}")
    if kt is torch.uint8 or kt is torch.float8_e4m3fn:
        want, dt = torch.bfloat16, DTYPE_BF16_KV_FP8
    elif kt is torch.bfloat16 or kt is torch.float32:
        want, dt = kt, DTYPE_BF16 if kt is torch.bfloat16 else DTYPE_F32
    else:
        raise ValueError(f"a cache must be bfloat16, float32 or FP8 codes, got {kt}")
    if q is not None and q.dtype is not want:
        raise ValueError(f"q must be {want} for a cache of {kt}, got {q.dtype}")
    return dt


def _lengths(t, b, what):
    if t is not None and (t.dtype is not torch.int32 or t.numel() != b):
        raise ValueError(f"{what} must be int32 [{b}]")
    return t


def _sums_ld(w, b, Hkv, P):
    """Elements between the rows of weights [b][Hkv][>= P] (float32, evenly spaced rows)."""
    if w.dtype is not torch.float32 or w.dim() != 3 or w.shape[0] != b or w.shape[1] != Hkv or w.shape[2] < P:
        raise ValueError(f"weights must be float32 [{b}][{Hkv}][>= {P}], got {w.dtype} {tuple(w.shape)}")
    sb, sh, sk = w.stride()
    ld = sh if Hkv > 1 else (sb if b > 1 else max(w.shape[2], 1))
    if (w.shape[2] > 1 and sk != 1) or (b > 1 and sb != Hkv * ld) or ld < P:
        raise ValueError("weights must have contiguous, evenly spaced rows")
    return ld


def dard_attention_shared_workspace_bytes(dtype, b, B, Hq, Hkv, dh, Ps, P):
    return lib().dard_attention_shared_workspace_bytes(dtype, b, B, Hq, Hkv, dh, Ps, P)


def dard_masked_attention_shared(q, k_shared, v_shared, Ps, k, v, P, state, conf, scale, flags, out, lse=None, ws=None,
                                 prefix=None, stream=None):
    """dard_masked_attention of a batch with Ps keys of a shared cache (k_shared [Hkv][cap_shared][dh], v_shared
    [Hkv][dh][cap_shared]; None where Ps is 0) before each sequence's own (k [b][Hkv][cap][dh], v [b][Hkv][dh][cap]:
    prefix[s] or P keys, then the block); lse: float32 [b][2B][Hq] or None."""
    b, R, Hq, dh = q.shape
    _, Hkv, cap, _ = k.shape
    if k.shape != (b, Hkv, cap, dh) or v.shape != (b, Hkv, dh, cap):
        raise ValueError(f"k must be [b][Hkv][cap][dh], v [b][Hkv][dh][cap], got {tuple(k.shape)} and {tuple(v.shape)}")
    cap_sh = 0
    if k_shared is not None or v_shared is not None:
        if k_shared is None or v_shared is None:
            raise ValueError("k_shared and v_shared go together")
        cap_sh = k_shared.shape[1]
        if k_shared.shape != (Hkv, cap_sh, dh) or v_shared.shape != (Hkv, dh, cap_sh):
            raise ValueError("k_shared must be [Hkv][cap_shared][dh], v_shared [Hkv][dh][cap_shared]")
    if out.shape != q.shape or out.dtype is not q.dtype:
        raise ValueError("out must be as q")
    if R % 2 or state.shape != (b, R // 2) or conf.shape != state.shape:
        raise ValueError(f"state and conf must be [b][B] = {(b, R // 2)}")
    if state.dtype is not torch.uint8 or conf.dtype is not torch.float32:
        raise ValueError("state must be uint8, conf float32")
    if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (b, R, Hq)):
        raise ValueError(f"lse must be float32 {(b, R, Hq)}")
    dt = _kv_dt(q, k, v, k_shared, v_shared)
    (qp, ks, vs, kp, vp, pre, sp, cp, op, lp, room), st = _args(
        stream, (q, k_shared, v_shared, k, v, _lengths(prefix, b, "prefix"), state, conf, out, lse, ws))
    _check(lib().dard_masked_attention_shared(dt, qp, ks, vs, Ps, cap_sh, kp, vp, P, pre, cap, sp, cp, b, R // 2, Hq, Hkv,
                                              dh, scale, flags, op, lp, room, _nbytes(ws), st))


def dard_key_weights_workspace_bytes(dtype, b, R, Hq, Hkv, dh, P):
    return lib().dard_key_weights_workspace_bytes(dtype, b, R, Hq, Hkv, dh, P)


def dard_key_weights(q, lse, k, P, scale, decay, weights, ws=None, prefix=None, stream=None):
    """weights [b][Hkv][>= P] (float32, rows may be further apart) = decay weights + the softmax weight of every prefix
    key of k [b][Hkv][cap][dh], summed over the rows q [b][R][Hq][dh] with lse [b][R][Hq]."""
    b, R, Hq, dh = q.shape
    _, Hkv, cap, _ = k.shape
    if k.shape != (b, Hkv, cap, dh):
        raise ValueError(f"k must be [b][Hkv][cap][dh], got {tuple(k.shape)}")
    if lse.dtype is not torch.float32 or lse.shape != (b, R, Hq):
        raise ValueError(f"lse must be float32 {(b, R, Hq)}")
    ld = _sums_ld(weights, b, Hkv, P)
    dt = _kv_dt(q, k)
    (qp, lp, kp, pre, room, wp), st = _args(stream, (q, lse, k, _lengths(prefix, b, "prefix"), ws), (weights,))
    _check(lib().dard_key_weights(dt, qp, lp, kp, P, pre, cap, b, R, Hq, Hkv, dh, scale, decay, wp, ld, room, _nbytes(ws),
                                  st))


def dard_kv_select_workspace_bytes(b, Hkv, P, n):
    return lib().dard_kv_select_workspace_bytes(b, Hkv, P, n)


def dard_kv_select(weights, P, keep, first=0, last=0, kept=None, ws=None, prefix=None, stream=None):
    """keep [b][Hkv][n] (int32): ascending indices of the keys of the largest weights [b][Hkv][>= P], the first and the
    last few always among them, -1 from kept[s] = min(n, prefix[s] or P) on; kept: int32 [b] or None."""
    if keep.dtype is not torch.int32 or keep.dim() != 3:
        raise ValueError("keep must be int32 [b][Hkv][n]")
    b, Hkv, n = keep.shape
    ld = _sums_ld(weights, b, Hkv, P)
    (kp, np_, pre, room, wp), st = _args(
        stream, (keep, _lengths(kept, b, "kept"), _lengths(prefix, b, "prefix"), ws), (weights,))
    _check(lib().dard_kv_select(wp, ld, P, pre, b, Hkv, n, first, last, kp, np_, room, _nbytes(ws), st))


def dard_kv_compact(k, v, keep, P, weights=None, kept=None, prefix=None, stream=None):
    """Keys keep[s][g][j] of k [b][Hkv][cap][dh], v [b][Hkv][dh][cap] and weights [b][Hkv][>= P] (or None) to places j <
    kept[s] (None: keep's n), in place; freed weights become 0."""
    b, Hkv, cap, dh = k.shape
    if v.shape != (b, Hkv, dh, cap):
        raise ValueError(f"v must be [b][Hkv][dh][cap] = {(b, Hkv, dh, cap)}, got {tuple(v.shape)}")
    if keep.dtype is not torch.int32 or keep.dim() != 3 or keep.shape[:2] != (b, Hkv):
        raise ValueError(f"keep must be int32 [{b}][{Hkv}][n]")
    dt = _kv_dt(None, k, v)
    ld = 0 if weights is None else _sums_ld(weights, b, Hkv, P)
    (kp, vp, ip, np_, pre, *w), st = _args(stream, (k, v, keep, _lengths(kept, b, "kept"), _lengths(prefix, b, "prefix")),
                                           () if weights is None else (weights,))
    _check(lib().dard_kv_compact(dt, kp, vp, cap, w[0] if w else None, ld, ip, keep.shape[2], np_, P, pre, b, Hkv, dh, st))


def dard_trace_enable(mask):
    _check(lib().dard_trace_enable(mask))


def dard_trace_read(cls):
    n = ctypes.c_int64(0)
    ms = ctypes.c_double(0.0)
    _check(lib().dard_trace_read(cls, ctypes.byref(n), ctypes.byref(ms)))
    return n.value, ms.value


def dard_trace_reset():
    _check(lib().dard_trace_reset())


def dard_trace_sample(period):
    _check(lib().dard_trace_sample(period))


def _debug(debug):
    if debug is None:
        return None
    return dard_step_debug(*[_p(debug.get(k)) for k in ("logits", "w", "maxprob_s", "argmax_s", "pcur_s",
                                                        "maxprob_mix", "argmax_mix", "entropy", "margin")])


class Engine:
    """Device state of one decoding job: packed weights, KV cache and
    workspace (torch allocations), plus calls of dard_prefill / dard_step."""

    def __init__(self, dims, weights, b, B, cap, stream=None, device="cuda", packed=None):
        """weights: name -> tensor (packed here), or None with `packed` = the
        packed image of another Engine of the same dims (shared, not copied)."""
        self.dims = dims
        self.cdims = make_dims(dims)
        self.b, self.B, self.cap = b, B, cap
        L = lib()
        nbytes = L.dard_packed_weight_bytes(ctypes.byref(self.cdims))
        if nbytes == 0:
            raise DardError(-2, L.dard_last_error().decode())
        if packed is not None:
            if packed.numel() < nbytes:
                raise ValueError("packed image too small for these dims")
            self.packed = packed
        else:
            self.packed = torch.empty(nbytes, dtype=torch.uint8, device=device)
            names = [n for n in weights]
            srcs = (ctypes.c_void_p * len(names))(*[_p(weights[n].contiguous()) for n in names])
            _check(L.dard_pack_weights(ctypes.byref(self.cdims), srcs, len(names), _p(self.packed), nbytes,
                                       _stream(stream)))
        kvb = L.dard_kv_bytes(ctypes.byref(self.cdims), b, cap)
        self.kv = torch.zeros(max(kvb, 16), dtype=torch.uint8, device=device)
        wsb = L.dard_workspace_bytes(ctypes.byref(self.cdims), b, B, cap)
        if wsb == 0:
            raise DardError(-2, L.dard_last_error().decode())
        self.ws = torch.zeros(wsb, dtype=torch.uint8, device=device)

    def kv_view(self, dtype):
        """KV cache as (K, V) tensors [layers][b][Hkv][cap][dh] (V read out of
        its dims-major storage [layers][b][Hkv][dh][cap] as a transposed view);
        dtype torch.uint8 for an FP8 cache (E4M3 codes)."""
        d = self.dims
        n = d.n_layers * 2 * self.b * d.n_kv_heads * self.cap * d.head_dim
        kv = self.kv.view(dtype)[:n].view(d.n_layers, 2, self.b, d.n_kv_heads, self.cap * d.head_dim)
        k = kv[:, 0].view(d.n_layers, self.b, d.n_kv_heads, self.cap, d.head_dim)
        v = kv[:, 1].view(d.n_layers, self.b, d.n_kv_heads, d.head_dim, self.cap).transpose(-1, -2)
        return k, v

    def dard_prefill(self, ids, embeds=None, stream=None):
        b, P = ids.shape
        _check(lib().dard_prefill(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap, b, P, _p(ids),
                                  _p(embeds), _p(self.ws), self.ws.numel(), _stream(stream)))

    def dard_step(self, P, params, tok_in, state_in, conf_in, tok_out, state_out, conf_out, block_done=None,
                  debug=None, stream=None):
        b, B = tok_in.shape
        dbg = None
        dbg = _debug(debug)
        _check(lib().dard_step(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap, P,
                               ctypes.byref(params), b, B, _p(tok_in), _p(state_in), _p(conf_in), _p(tok_out),
                               _p(state_out), _p(conf_out), _p(block_done), _ref(dbg), _p(self.ws),
                               self.ws.numel(), _stream(stream)))

    def dard_prefill_extend(self, P, ids, stream=None):
        """Extend-only refresh: positions P..P+Pn-1 of each sequence (ids
        [b][Pn]) see the cached keys 0..P-1 and each other."""
        b, Pn = ids.shape
        _check(lib().dard_prefill_extend(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap, P, b, Pn,
                                         _p(ids), _p(self.ws), self.ws.numel(), _stream(stream)))

    def dard_prefill_suffix(self, shared, Ps, ids, stream=None):
        """Positions Ps.. of each sequence after the prompt cached in `shared`
        (an Engine of the same dims with b = 1 whose dard_prefill ran over Ps
        prompt positions); ids [b][Pc]."""
        b, Pc = ids.shape
        _check(lib().dard_prefill_suffix(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap,
                                         _p(shared.kv), shared.cap, Ps, b, Pc, _p(ids), _p(self.ws), self.ws.numel(),
                                         _stream(stream)))

    def dard_step_shared(self, shared, Ps, P, params, tok_in, state_in, conf_in, tok_out, state_out, conf_out,
                         block_done=None, debug=None, stream=None):
        b, B = tok_in.shape
        dbg = _debug(debug)
        _check(lib().dard_step_shared(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap,
                                      _p(shared.kv), shared.cap, Ps, P, ctypes.byref(params), b, B, _p(tok_in),
                                      _p(state_in), _p(conf_in), _p(tok_out), _p(state_out), _p(conf_out),
                                      _p(block_done), _ref(dbg), _p(self.ws), self.ws.numel(), _stream(stream)))

    def dard_step_full(self, blk, params, seq, state_in, conf_in, tok_out, state_out, conf_out, block_done=None,
                       debug=None, stream=None):
        """Full-sequence step: seq [b][N] (current block at blk..blk+B-1)."""
        b, N = seq.shape
        B = state_in.shape[1]
        dbg = _debug(debug)
        _check(lib().dard_step_full(ctypes.byref(self.cdims), _p(self.packed), _p(self.kv), self.cap, N, blk,
                                    ctypes.byref(params), b, B, _p(seq), _p(state_in), _p(conf_in), _p(tok_out),
                                    _p(state_out), _p(conf_out), _p(block_done), _ref(dbg), _p(self.ws),
                                    self.ws.numel(), _stream(stream)))
