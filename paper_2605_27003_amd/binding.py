"""ctypes binding of include/svdq.h for torch tensors (device memory and streams only)."""
import array
import collections
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsvdq.so")
_lib = None

OUT_BF16, OUT_F32 = 0, 1
_vp, _i64, _i32, _f32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float

EXPORTS = {
    "svdq_status_string": (ctypes.c_char_p, [_i32]),
    "svdq_version": (_i32, []),
    "svdq_alpha_lookup": (_f32, [_vp, _i32, _i32, _i32, _i32]),
    "svdq_packed_l1_bytes": (ctypes.c_size_t, [_i32]),
    "svdq_pack_lowrank_down": (_i32, [_vp, _vp, _i32, _i32, _vp, _vp]),
    "svdq_quantize_act": (_i32, [_vp, _i64, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "svdq_packed_weight_bytes": (ctypes.c_size_t, [_i32, _i32]),
    "svdq_pack_weight": (_i32, [_vp, _vp, _i32, _i32, _vp, _vp]),
    "svdq_linear_w4a4": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _i64, _i32, _vp]),
    "svdq_lowrank": (_i32, [_i32, _vp, _i64, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _vp, _i64, _vp]),
    "svdq_act_e3m2_bytes": (ctypes.c_size_t, [_i64, _i32]),
    "svdq_quantize_act_e3m2": (_i32, [_vp, _i64, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "svdq_unpack_act_e3m2": (_i32, [_vp, _i64, _i32, _vp, _vp]),
    "svdq_packed_weight_e3m2_bytes": (ctypes.c_size_t, [_i32, _i32]),
    "svdq_pack_weight_e3m2": (_i32, [_vp, _vp, _i32, _i32, _vp, _vp]),
    "svdq_linear_w4a4_e3m2": (_i32, [_vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _i64, _i32, _vp]),
    "svdq_linear_w4a4_e3m2_next": (_i32, [_vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _i32,
                                          _vp, _f32, _vp, _i32, _vp, _vp, _vp, _vp]),
    "svdq_debug_group_acc_e3m2": (_i32, [_vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp, _vp]),
    "svdq_quantize_act_gelu": (_i32, [_i32, _vp, _i64, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "svdq_debug_gelu": (_i32, [_vp, _i64, _vp, _vp]),
    "svdq_quantize_act_mxfp4": (_i32, [_vp, _i64, _vp, _f32, _vp, _i64, _i32, _i32, _vp, _vp, _vp, _vp]),
    "svdq_packed_weight_mxfp4_bytes": (ctypes.c_size_t, [_i32, _i32]),
    "svdq_pack_weight_mxfp4": (_i32, [_vp, _vp, _i32, _i32, _vp, _vp]),
    "svdq_linear_mxfp4": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _vp, _i64, _i32, _vp]),
    "svdq_linear_mxfp4_next": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _i32, _i32,
                                      _vp, _f32, _vp, _i32, _vp, _vp, _vp, _vp]),
    "svdq_layer_codes_bytes": (ctypes.c_size_t, [_vp, _i64]),
    "svdq_layer_scratch_bytes": (ctypes.c_size_t, [_vp, _i64]),
    "svdq_layer_staging_bytes": (ctypes.c_size_t, [_vp, _i64]),
    "svdq_layer_forward": (_i32, [_vp, _vp, _i64, _f32, _i32, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _i64, _vp]),
    "svdq_layer_gemm": (_i32, [_vp, _vp, _vp, _vp, _i64, _vp, _vp, _i64, _vp]),
    "svdq_gptq_workspace_bytes": (ctypes.c_size_t, [_i32, _i32]),
    "svdq_gptq_hessian": (_i32, [_vp, _i64, _vp, _i64, _i32, _vp, _vp]),
    "svdq_gptq_quantize": (_i32, [_vp, _vp, ctypes.c_double, _i32, _i32, _vp, _vp, _vp, _vp]),
    "svdq_sq_error_workspace_bytes": (ctypes.c_size_t, []),
    "svdq_sq_error": (_i32, [_vp, _i64, _vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "svdq_sq_error_add": (_i32, [_vp, _i64, _vp, _i64, _i64, _i32, _vp, _vp, _vp]),
    "svdq_argmin_rows": (_i32, [_vp, _i32, _i32, _vp, _vp]),
    "svdq_sq_error_static": (_i32, [_vp, _i64, _vp, _i64, _i64, _i32, _vp, _vp]),
    "svdq_quantize_act_int8": (_i32, [_vp, _i64, _vp, _f32, _i32, _i64, _i32, _vp, _vp, _vp]),
    "svdq_linear_w8a8": (_i32, [_vp, _vp, _vp, _vp, _vp, _i64, _i32, _i32, _vp, _i64, _i32, _vp]),
    "svdq_quantize_act_int8_grouped": (_i32, [_vp, _i64, _i64, _vp, _vp, _i32, _vp, _f32, _vp, _i32, _i64, _i32, _vp, _vp, _vp]),
    "svdq_linear_w8a8_grouped": (_i32, [_vp, _vp, _vp, _vp, _vp, _vp, _i32, _i64, _i32, _i32, _vp, _i64, _i32, _vp]),
    "svdq_layer_int8_rows_on_chip": (_i64, [_vp]),
    "svdq_layer_int8_forward": (_i32, [_vp, _vp, _i64, _i64, _vp, _vp, _f32, _vp, _i32, _i64, _vp, _vp, _vp, _i64, _vp]),
    "svdq_debug_group_acc": (_i32, [_vp, _vp, _i64, _i32, _i32, _i64, _i32, _vp, _vp]),
    "svdq_debug_scale_chain": (_i32, [_vp, _f32, _i64, _vp, _vp, _vp]),
}


class SvdqError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {load_library().svdq_status_string(status).decode()} ({status})")


def load_library(build_if_missing=True):
    """Load libsvdq.so (built in-tree by paper_2605_27003_amd/build.py); never falls back to anything else."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            if not build_if_missing:
                raise FileNotFoundError(_LIB_PATH)
            from . import build as _build
            _build.build(force=True)
        lib = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


# hipStream_t of the current stream of the current device.  torch.cuda.current_stream() builds a Stream object for it:
# 2.8 us against 0.1 us, of the 12 us that the host needs for a layer with few tokens.  Where torch has renamed its own
# functions, the public way.
def _raw_stream():
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:
        return torch.cuda.current_stream().cuda_stream


def _stream():
    return ctypes.c_void_p(_raw_stream())


def _check(rc, where):
    if rc != 0:
        raise SvdqError(rc, where)


def version():
    return int(load_library().svdq_version())


def alpha_lookup(table, step, step0, nsteps_expert):
    arr = array.array("f", [*table])
    return (_lib or load_library()).svdq_alpha_lookup(arr.buffer_info()[0], len(arr), step, step0, nsteps_expert)


def packed_l1_bytes(K):
    return int(load_library().svdq_packed_l1_bytes(K))


def packed_weight_bytes(N, K):
    return int(load_library().svdq_packed_weight_bytes(N, K))


def pack_lowrank_down(L1_bf16, inv_lambda):
    """L1 [K,r] bf16, inv_lambda [K] f32 (device) -> opaque uint8 tensor for quantize_act."""
    K, r = L1_bf16.shape
    out = torch.empty(packed_l1_bytes(K), dtype=torch.uint8, device=L1_bf16.device)
    _check(load_library().svdq_pack_lowrank_down(_ptr(L1_bf16), _ptr(inv_lambda), K, r, _ptr(out), _stream()),
           "svdq_pack_lowrank_down")
    return out


def pack_weight(qw, sw):
    """qw [N,K/2] uint8 canonical codes, sw [K/64,N] f32 (device) -> opaque uint8 tensor for linear_w4a4."""
    N, K2 = qw.shape
    K = 2 * K2
    out = torch.empty(packed_weight_bytes(N, K), dtype=torch.uint8, device=qw.device)
    _check(load_library().svdq_pack_weight(_ptr(qw), _ptr(sw), N, K, _ptr(out), _stream()), "svdq_pack_weight")
    return out


def quantize_act(x_bf16, inv_lambda, rho, l1_packed=None, r=0, out=None):
    """x [M,K] bf16 (row stride allowed) -> (qx [K/64,M,32] u8, sx [K/64,M] f32, h [M,r] f32 or None).

    qx and sx are group-major (see include/svdq.h); `to_token_major` gives the [M,K/2] / [M,K/64] view."""
    M, K = x_bf16.shape
    assert x_bf16.dtype == torch.bfloat16 and x_bf16.stride(1) == 1
    dev = x_bf16.device
    if out is None:
        qx = torch.empty((K // 64, M, 32), dtype=torch.uint8, device=dev)
        sx = torch.empty((K // 64, M), dtype=torch.float32, device=dev)
        h = torch.empty((M, r), dtype=torch.float32, device=dev) if l1_packed is not None else None
    else:
        qx, sx, h = out
    ldx = x_bf16.stride(0) if M > 1 else K
    _check(load_library().svdq_quantize_act(_ptr(x_bf16), ldx, _ptr(inv_lambda), float(rho), _ptr(l1_packed),
                                           M, K, r if l1_packed is not None else 0,
                                           _ptr(qx), _ptr(sx), _ptr(h), _stream()), "svdq_quantize_act")
    return qx, sx, h


def to_token_major(qx, sx):
    """Group-major (qx [K/64,M,32], sx [K/64,M]) -> token-major copies (qx [M,K/2], sx [M,K/64])."""
    ng, M, _ = qx.shape
    return qx.permute(1, 0, 2).reshape(M, ng * 32).contiguous(), sx.t().contiguous()


def to_group_major(qx_tm, sx_tm):
    """Token-major (qx [M,K/2], sx [M,K/64]) -> group-major copies, the layout the GEMM consumes."""
    M, K2 = qx_tm.shape
    return qx_tm.reshape(M, K2 // 32, 32).permute(1, 0, 2).contiguous(), sx_tm.t().contiguous()


def linear_w4a4(qx, sx, w_packed, N, h=None, L2_bf16=None, bias=None, out=None, out_dtype=torch.bfloat16):
    """qx [K/64,M,32], sx [K/64,M] (group-major) -> y [M,N] bf16 (or f32: the value before the bf16 rounding)."""
    ng, M, _ = qx.shape
    K = 64 * ng
    r = 0 if h is None else h.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=qx.device)
    code = OUT_F32 if out.dtype == torch.float32 else OUT_BF16
    ldy = out.stride(0) if M > 1 else N
    _check(load_library().svdq_linear_w4a4(_ptr(qx), _ptr(sx), _ptr(w_packed), _ptr(h), _ptr(L2_bf16), _ptr(bias),
                                          M, N, K, r, _ptr(out), ldy, code, _stream()), "svdq_linear_w4a4")
    return out


def lowrank(mode, *, x_bf16=None, inv_lambda=None, L_bf16=None, h=None, y_bf16=None):
    """mode 0: h = (x*inv_lambda) L1 (returns h); mode 1: y += h L2 in place (returns y)."""
    lib = load_library()
    if mode == 0:
        M, K = x_bf16.shape
        r = L_bf16.shape[1]
        if h is None:
            h = torch.empty((M, r), dtype=torch.float32, device=x_bf16.device)
        ldx = x_bf16.stride(0) if M > 1 else K
        _check(lib.svdq_lowrank(0, _ptr(x_bf16), ldx, _ptr(inv_lambda), _ptr(L_bf16), M, K, 0, r,
                                _ptr(h), None, 0, _stream()), "svdq_lowrank")
        return h
    M, N = y_bf16.shape
    r = L_bf16.shape[0]
    ldy = y_bf16.stride(0) if M > 1 else N
    _check(lib.svdq_lowrank(1, None, 0, None, _ptr(L_bf16), M, 0, N, r, _ptr(h), _ptr(y_bf16), ldy, _stream()),
           "svdq_lowrank")
    return y_bf16


def debug_group_acc(qx, w_packed, N, m0, mt):
    """int32 group accumulators of rows [m0, m0+mt) as the GEMM kernel forms them -> [mt, N, K/64]."""
    ng, M, _ = qx.shape
    K = 64 * ng
    acc = torch.empty((mt, N, K // 64), dtype=torch.int32, device=qx.device)
    _check(load_library().svdq_debug_group_acc(_ptr(qx), _ptr(w_packed), M, N, K, m0, mt, _ptr(acc), _stream()),
           "svdq_debug_group_acc")
    return acc


# ---- E3M2-container execution of the int4 layer -------------------------------------------------
class ActE3M2(collections.namedtuple("ActE3M2", "buf M K")):
    """Activation operand buffer of the FP6 matrix-core path (layout in include/svdq.h) with its logical shape."""


def act_e3m2_bytes(M, K):
    return load_library().svdq_act_e3m2_bytes(M, K)


def quantize_act_e3m2(x_bf16, inv_lambda, rho, l1_packed=None, r=0, out=None, want_sx=True):
    """x [M,K] bf16 -> (act ActE3M2, sx [K/64,M] f32 or None, h [M,r] f32 or None).  Same codes and scales as
    quantize_act, codes held as E3M2 fields."""
    M, K = x_bf16.shape
    assert x_bf16.dtype == torch.bfloat16 and x_bf16.stride(1) == 1
    dev = x_bf16.device
    if out is None:
        act = ActE3M2(torch.empty(act_e3m2_bytes(M, K), dtype=torch.uint8, device=dev), M, K)
        sx = torch.empty((K // 64, M), dtype=torch.float32, device=dev) if want_sx else None
        h = torch.empty((M, r), dtype=torch.float32, device=dev) if l1_packed is not None else None
    else:
        act, sx, h = out
        assert act.M == M and act.K == K
    ldx = x_bf16.stride(0) if M > 1 else K
    _check(load_library().svdq_quantize_act_e3m2(_ptr(x_bf16), ldx, _ptr(inv_lambda), float(rho), _ptr(l1_packed),
                                                M, K, r if l1_packed is not None else 0,
                                                _ptr(act.buf), _ptr(sx), _ptr(h), _stream()), "svdq_quantize_act_e3m2")
    return act, sx, h


def unpack_act_e3m2(act):
    """ActE3M2 -> nibble codes qx [K/64,M,32] u8 in the layout of quantize_act."""
    qx = torch.empty((act.K // 64, act.M, 32), dtype=torch.uint8, device=act.buf.device)
    _check(load_library().svdq_unpack_act_e3m2(_ptr(act.buf), act.M, act.K, _ptr(qx), _stream()), "svdq_unpack_act_e3m2")
    return qx


def packed_weight_e3m2_bytes(N, K):
    return load_library().svdq_packed_weight_e3m2_bytes(N, K)


def pack_weight_e3m2(qw, sw, out=None):
    """qw [N,K/2] uint8 canonical codes, sw [K/64,N] f32 (device) -> opaque uint8 tensor for linear_w4a4_e3m2.
    `out`: a caller's buffer of at least packed_weight_e3m2_bytes(N, K) bytes (e.g. one staging buffer shared by
    every layer of a model whose weights stay resident in the canonical 4-bit form)."""
    N, K2 = qw.shape
    K = 2 * K2
    if out is None:
        out = torch.empty(packed_weight_e3m2_bytes(N, K), dtype=torch.uint8, device=qw.device)
    assert out.numel() >= packed_weight_e3m2_bytes(N, K)
    _check(load_library().svdq_pack_weight_e3m2(_ptr(qw), _ptr(sw), N, K, _ptr(out), _stream()), "svdq_pack_weight_e3m2")
    return out


def linear_w4a4_e3m2(act, w_packed, N, h=None, L2_bf16=None, bias=None, out=None, out_dtype=torch.bfloat16):
    """ActE3M2 -> y [M,N] bf16 (or f32: the value before the bf16 rounding)."""
    M, K = act.M, act.K
    r = 0 if h is None else h.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=act.buf.device)
    code = OUT_F32 if out.dtype == torch.float32 else OUT_BF16
    ldy = out.stride(0) if M > 1 else N
    _check(load_library().svdq_linear_w4a4_e3m2(_ptr(act.buf), _ptr(w_packed), _ptr(h), _ptr(L2_bf16), _ptr(bias),
                                               M, N, K, r, _ptr(out), ldy, code, _stream()), "svdq_linear_w4a4_e3m2")
    return out


def linear_w4a4_e3m2_next(act, w_packed, N, next_inv_lambda, next_rho, h=None, L2_bf16=None, bias=None, gelu=True,
                          next_l1_packed=None, next_r=0, out=None, want_sx=True):
    """The layer on `act` fused with the NEXT layer's quantise pass (optionally through GELU): returns what
    quantize_act_e3m2 / quantize_act_gelu(FMT_INT4_E3M2) of this layer's bf16 output would return,
    (ActE3M2 of shape [M, N], sx [N/64, M] or None, h' [M, next_r] or None), without y ever being stored."""
    M, K = act.M, act.K
    r = 0 if h is None else h.shape[1]
    dev = act.buf.device
    if out is None:
        nact = ActE3M2(torch.empty(act_e3m2_bytes(M, N), dtype=torch.uint8, device=dev), M, N)
        nsx = torch.empty((N // 64, M), dtype=torch.float32, device=dev) if want_sx else None
        nh = torch.empty((M, next_r), dtype=torch.float32, device=dev) if next_l1_packed is not None else None
    else:
        nact, nsx, nh = out
        assert nact.M == M and nact.K == N
    _check(load_library().svdq_linear_w4a4_e3m2_next(
        _ptr(act.buf), _ptr(w_packed), _ptr(h), _ptr(L2_bf16), _ptr(bias), M, N, K, r, int(bool(gelu)),
        _ptr(next_inv_lambda), float(next_rho), _ptr(next_l1_packed), next_r if next_l1_packed is not None else 0,
        _ptr(nact.buf), _ptr(nsx), _ptr(nh), _stream()), "svdq_linear_w4a4_e3m2_next")
    return nact, nsx, nh


def debug_group_acc_e3m2(act, w_packed, N, m0, mt):
    """Integer group sums of rows [m0, m0+mt) as the FP6 matrix-core path forms them -> [mt, N, K/64] int32."""
    acc = torch.empty((mt, N, act.K // 64), dtype=torch.int32, device=act.buf.device)
    _check(load_library().svdq_debug_group_acc_e3m2(_ptr(act.buf), _ptr(w_packed), act.M, N, act.K, m0, mt,
                                                   _ptr(acc), _stream()), "svdq_debug_group_acc_e3m2")
    return acc


# ---- kernel (a) with GELU fused ----------------------------------------------------------------
FMT_INT4, FMT_INT4_E3M2, FMT_MXFP4 = 0, 1, 2


def quantize_act_gelu(fmt, x_bf16, inv_lambda, rho, l1_packed=None, r=0, out=None):
    """quantize_act / quantize_act_e3m2 / quantize_act_mxfp4 (fmt = FMT_*) of gelu(x), the activation applied on the
    fly; returns what that function returns."""
    M, K = x_bf16.shape
    assert x_bf16.dtype == torch.bfloat16 and x_bf16.stride(1) == 1
    dev = x_bf16.device
    if out is None:
        h = torch.empty((M, r), dtype=torch.float32, device=dev) if l1_packed is not None else None
        if fmt == FMT_INT4_E3M2:
            codes = ActE3M2(torch.empty(act_e3m2_bytes(M, K), dtype=torch.uint8, device=dev), M, K)
            scales = torch.empty((K // 64, M), dtype=torch.float32, device=dev)
        else:
            codes = torch.empty((K // 64, M, 32), dtype=torch.uint8, device=dev)
            scales = (torch.empty((K // 64, M), dtype=torch.float32, device=dev) if fmt == FMT_INT4
                      else torch.empty(((K // 64 + 1) // 2, M, 2, 2), dtype=torch.uint8, device=dev))
    else:
        codes, scales, h = out
    buf = codes.buf if fmt == FMT_INT4_E3M2 else codes
    ldx = x_bf16.stride(0) if M > 1 else K
    _check(load_library().svdq_quantize_act_gelu(fmt, _ptr(x_bf16), ldx, _ptr(inv_lambda), float(rho), _ptr(l1_packed),
                                                M, K, r if l1_packed is not None else 0,
                                                _ptr(buf), _ptr(scales), _ptr(h), _stream()), "svdq_quantize_act_gelu")
    return codes, scales, h


def debug_gelu(x_bf16):
    """bf16 tensor -> bf16(gelu(x)) through the device function of the fused quantise pass."""
    x = x_bf16.contiguous()
    out = torch.empty_like(x)
    _check(load_library().svdq_debug_gelu(_ptr(x), x.numel(), _ptr(out), _stream()), "svdq_debug_gelu")
    return out


# ---- GPTQ on the residual (offline calibration) ------------------------------------------------
def gptq_hessian(x_bf16, inv_lambda, H=None):
    """H [K,K] f64 += X^T X^ over the rows of x (a new zero H if none is given)."""
    M, K = x_bf16.shape
    if H is None:
        H = torch.zeros((K, K), dtype=torch.float64, device=x_bf16.device)
    ldx = x_bf16.stride(0) if M > 1 else K
    _check(load_library().svdq_gptq_hessian(_ptr(x_bf16), ldx, _ptr(inv_lambda), M, K, _ptr(H), _stream()), "svdq_gptq_hessian")
    return H


def gptq_quantize(R_f32, H_f64, damp=0.01):
    """R [K,N] f32 residual, H [K,K] f64 -> (qw [N,K/2] u8 canonical codes, sw [K/64,N] f32 scales)."""
    K, N = R_f32.shape
    dev = R_f32.device
    ws = torch.empty(load_library().svdq_gptq_workspace_bytes(N, K), dtype=torch.uint8, device=dev)
    qw = torch.empty((N, K // 2), dtype=torch.uint8, device=dev)
    sw = torch.empty((K // 64, N), dtype=torch.float32, device=dev)
    _check(load_library().svdq_gptq_quantize(_ptr(R_f32.contiguous()), _ptr(H_f64.contiguous()), float(damp), N, K,
                                            _ptr(ws), _ptr(qw), _ptr(sw), _stream()), "svdq_gptq_quantize")
    return qw, sw


# ---- MXFP4 variant ---------------------------------------------------------------------------
def quantize_act_mxfp4(x_bf16, inv_lambda, rho, l1_packed=None, r=0, out=None):
    """x [M,K] bf16 -> (qx [K/64,M,32] u8 E2M1 codes, sx [ceil(K/128),M,2,2] u8 E8M0 bytes, h [M,r] f32 or None)."""
    M, K = x_bf16.shape
    ldx = x_bf16.stride(0) if M > 1 else K
    if out is None:
        qx = torch.empty((K // 64, M, 32), dtype=torch.uint8, device=x_bf16.device)
        sx = torch.empty(((K // 64 + 1) // 2, M, 2, 2), dtype=torch.uint8, device=x_bf16.device)
        h = torch.empty((M, r), dtype=torch.float32, device=x_bf16.device) if l1_packed is not None else None
    else:
        qx, sx, h = out
    _check(load_library().svdq_quantize_act_mxfp4(_ptr(x_bf16), ldx, _ptr(inv_lambda), float(rho), _ptr(l1_packed),
                                                  M, K, r if l1_packed is not None else 0,
                                                  _ptr(qx), _ptr(sx), _ptr(h), _stream()), "svdq_quantize_act_mxfp4")
    return qx, sx, h


def mx_to_token_major(qx, sx, K):
    """Group-major MXFP4 activations -> (qx [M,K/2], sx [M,K/32]): the layout the format's definition suggests."""
    ng, M, _ = qx.shape
    qx_tm = qx.permute(1, 0, 2).reshape(M, ng * 32).contiguous()
    # sx[s][m][h][j] scales MX block 2 (2s + j) + h  ->  [m][s][j][h]
    sx_tm = sx.permute(1, 0, 3, 2).reshape(M, -1)[:, : K // 32].contiguous()
    return qx_tm, sx_tm


def packed_weight_mxfp4_bytes(N, K):
    return int(load_library().svdq_packed_weight_mxfp4_bytes(N, K))


def pack_weight_mxfp4(qw, sw):
    """qw [N,K/2] u8 packed E2M1 codes, sw [K/32,N] u8 E8M0 bytes (device) -> opaque uint8 tensor for linear_mxfp4."""
    N, K2 = qw.shape
    K = 2 * K2
    out = torch.empty(packed_weight_mxfp4_bytes(N, K), dtype=torch.uint8, device=qw.device)
    _check(load_library().svdq_pack_weight_mxfp4(_ptr(qw), _ptr(sw), N, K, _ptr(out), _stream()), "svdq_pack_weight_mxfp4")
    return out


def linear_mxfp4(qx, sx, w_packed, N, h=None, L2_bf16=None, bias=None, out=None, out_dtype=torch.bfloat16):
    """MXFP4 layer from quantised activations -> y [M,N] bf16 (or f32: the value before the bf16 rounding)."""
    ng, M, _ = qx.shape
    K = 64 * ng
    r = 0 if h is None else h.shape[1]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=qx.device)
    code = OUT_F32 if out.dtype == torch.float32 else OUT_BF16
    ldy = out.stride(0) if M > 1 else N
    _check(load_library().svdq_linear_mxfp4(_ptr(qx), _ptr(sx), _ptr(w_packed), _ptr(h), _ptr(L2_bf16), _ptr(bias),
                                            M, N, K, r, _ptr(out), ldy, code, _stream()), "svdq_linear_mxfp4")
    return out


def linear_mxfp4_next(qx, sx, w_packed, N, next_inv_lambda, next_rho, h=None, L2_bf16=None, bias=None, gelu=True,
                      next_l1_packed=None, next_r=0, out=None):
    """The MXFP4 layer fused with the NEXT layer's quantise pass (optionally through GELU): returns what
    quantize_act_mxfp4 / quantize_act_gelu(FMT_MXFP4) of this layer's bf16 output would return
    (qx' [N/64,M,32], sx' [N/128,M,2,2], h' [M,next_r] or None), without y ever being stored."""
    ng, M, _ = qx.shape
    K = 64 * ng
    r = 0 if h is None else h.shape[1]
    if out is None:
        nq = torch.empty((N // 64, M, 32), dtype=torch.uint8, device=qx.device)
        ns = torch.empty((N // 128, M, 2, 2), dtype=torch.uint8, device=qx.device)
        nh = torch.empty((M, next_r), dtype=torch.float32, device=qx.device) if next_l1_packed is not None else None
    else:
        nq, ns, nh = out
    _check(load_library().svdq_linear_mxfp4_next(
        _ptr(qx), _ptr(sx), _ptr(w_packed), _ptr(h), _ptr(L2_bf16), _ptr(bias), M, N, K, r, int(bool(gelu)),
        _ptr(next_inv_lambda), float(next_rho), _ptr(next_l1_packed), next_r if next_l1_packed is not None else 0,
        _ptr(nq), _ptr(ns), _ptr(nh), _stream()), "svdq_linear_mxfp4_next")
    return nq, ns, nh


# ---- clipping-ratio search (offline calibration, Sec. III-C) ---------------------------------
def sq_error(y_ref, y, workspace=None, out=None):
    """sum (y_ref - y)^2 over two bf16 [M,N] tensors -> 1-element float64 device tensor."""
    M, N = y.shape
    if workspace is None:
        workspace = torch.empty(load_library().svdq_sq_error_workspace_bytes() // 8, dtype=torch.float64, device=y.device)
    if out is None:
        out = torch.empty(1, dtype=torch.float64, device=y.device)
    _check(load_library().svdq_sq_error(_ptr(y_ref), y_ref.stride(0) if M > 1 else N, _ptr(y), y.stride(0) if M > 1 else N,
                                        M, N, _ptr(workspace), _ptr(out), _stream()), "svdq_sq_error")
    return out


def sq_error_static(y_ref, y, out=None):
    """sq_error through the entry point that allocates nothing and takes no workspace (partial sums in the
    library's static device array)."""
    M, N = y.shape
    if out is None:
        out = torch.empty(1, dtype=torch.float64, device=y.device)
    _check(load_library().svdq_sq_error_static(_ptr(y_ref), y_ref.stride(0) if M > 1 else N, _ptr(y),
                                               y.stride(0) if M > 1 else N, M, N, _ptr(out), _stream()),
           "svdq_sq_error_static")
    return out


def search_clipping_ratios(layer_run, xs, y_refs, bins, nbins, candidates):
    """Timestep-bin clipping-ratio search.  `layer_run(x, rho)` runs the quantised layer (quantise + GEMM kernels)
    and returns y bf16; xs[i], y_refs[i] are the calibration input and full-precision output of step i, bins[i]
    its timestep bin.  Returns (table [nbins] of chosen ratios, err [nbins][len(candidates)] summed errors).
    The sums over a bin's steps and the arg-min over the candidates run in the library, on the device."""
    lib = load_library()
    dev = xs[0].device
    nc = len(candidates)
    ws = torch.empty(lib.svdq_sq_error_workspace_bytes() // 8, dtype=torch.float64, device=dev)
    acc = torch.zeros((nbins, nc), dtype=torch.float64, device=dev)
    idx = torch.empty(nbins, dtype=torch.int32, device=dev)
    for x, yr, b in zip(xs, y_refs, bins):
        M, N = yr.shape
        for ci, rho in enumerate(candidates):
            y = layer_run(x, rho)
            _check(lib.svdq_sq_error_add(_ptr(yr), yr.stride(0) if M > 1 else N, _ptr(y), y.stride(0) if M > 1 else N,
                                         M, N, _ptr(ws), ctypes.c_void_p(acc.data_ptr() + 8 * (b * nc + ci)), _stream()),
                   "svdq_sq_error_add")
    _check(lib.svdq_argmin_rows(_ptr(acc), nbins, nc, _ptr(idx), _stream()), "svdq_argmin_rows")
    table = [float(candidates[i]) for i in idx.cpu().tolist()]
    return table, acc.cpu().numpy()


def debug_scale_chain(a, rho):
    """(s, 1/s) of eq. 8-9 for group magnitudes a (float32 device tensor), from the kernel's device functions."""
    a = a.contiguous()
    s = torch.empty_like(a)
    inv = torch.empty_like(a)
    _check(load_library().svdq_debug_scale_chain(_ptr(a), float(rho), a.numel(), _ptr(s), _ptr(inv), _stream()),
           "svdq_debug_scale_chain")
    return s, inv


_staging = {}        # device -> uint8 tensor shared by every W4A4Linear that keeps its weights in the canonical form


def _staging_buffer(nbytes, device):
    buf = _staging.get(device)
    if buf is None or buf.numel() < nbytes:
        buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _staging[device] = buf
    return buf


class _Layer(ctypes.Structure):
    """svdq_layer of include/svdq.h."""
    _fields_ = ([(n, _i32) for n in ("format", "N", "K", "r")] +
                [(n, _vp) for n in ("inv_lambda", "l1_packed", "L2_bf16", "bias", "w_packed", "qw", "sw")])


# One layer's buffers for one token count: the library's view (ptrs: codes, sx, h, scratch; bytes of staging, shared or
# not), the caller's (public), what they were made for (key) and the descriptor that they were last used with.
_Work = collections.namedtuple("_Work", "codes sx h scratch staging shared y public ptrs y_ptr key layer")


def _addr(t):
    return None if t is None else t.data_ptr()


_FORMATS = {"e3m2": FMT_INT4_E3M2, "nibble": FMT_INT4, "mxfp4": FMT_MXFP4}


class W4A4Linear:
    """One quantised linear resident in HBM: weights and low-rank factors, reusable output buffers.

    container "e3m2" (default) runs the int4 layer on the FP6 matrix cores, "nibble" the same layer from 4-bit packed
    weights (quantize() and gemm() on 4-bit activations and the int8 matrix cores; forward() on the FP6 ones, with the
    same codes and scales), "mxfp4" the MXFP4 format (qw then holds E2M1 codes and sw [K/32, N] E8M0 bytes).
    resident "w4" (default, container "e3m2" only) keeps the canonical 4-bit weights (qw, sw) and expands them into a
    staging buffer shared by all such layers of the device right before a GEMM of many tokens (calls on one stream only;
    where weights could also be expanded in registers the memory is taken for the call alone, so that any streams do);
    "packed" keeps the container's own packed form (7 - 8 bits per weight for the int4 containers), and forward() of the
    nibble container takes the memory that it expands weights and codes into for the call alone, from torch's allocator.
    buffers() holds, after quantize() as after forward(), what the container's quantise pass wrote."""

    def __init__(self, inv_lambda, L1_bf16, L2_bf16, qw, sw, bias, container="e3m2", resident="w4"):
        assert container in ("e3m2", "nibble", "mxfp4") and resident in ("w4", "packed")
        self.container = container
        self.format = _FORMATS[container]
        self.N, self.K = qw.shape[0], qw.shape[1] * 2
        self.r = 0 if L1_bf16 is None else L1_bf16.shape[1]
        self.inv_lambda = inv_lambda
        self.l1_packed = pack_lowrank_down(L1_bf16, inv_lambda) if self.r else None
        self.L2 = L2_bf16 if self.r else None
        self.qw = self.sw = None
        if container == "e3m2" and resident == "w4":
            self.qw, self.sw, self.w_packed = qw, sw, None
        else:
            self.w_packed = {"e3m2": pack_weight_e3m2, "nibble": pack_weight, "mxfp4": pack_weight_mxfp4}[container](qw, sw)
        self.bias = bias
        self._work = self._layer = None

    def _descriptor(self, r):
        """svdq_layer of the tensors that the layer holds now (they may have been replaced), with rank r.  The caller keeps
        it through its call: another thread may take the layer's place for one of its own meanwhile."""
        l1, L2, bias, wp, qw, sw = self.l1_packed, self.L2, self.bias, self.w_packed, self.qw, self.sw
        fields = (self.format, self.N, self.K, r, self.inv_lambda.data_ptr(),
                  None if l1 is None else l1.data_ptr(), None if L2 is None else L2.data_ptr(), None if bias is None else bias.data_ptr(),
                  None if wp is None else wp.data_ptr(), None if qw is None else qw.data_ptr(), None if sw is None else sw.data_ptr())
        layer = self._layer
        if layer is None or layer.values != fields:
            layer = _Layer(*fields)
            layer.values, layer.address = fields, ctypes.addressof(layer)
            self._layer = layer
        return layer

    def __getstate__(self):
        """Copies make buffers and a descriptor of their own."""
        return {**self.__dict__, "_work": None, "_layer": None}

    def __setstate__(self, state):
        """Also of layers saved with their buffers, and before the format code and the canonical tensors were attributes."""
        self.__dict__.update({"qw": None, "sw": None, **state, "format": _FORMATS[state["container"]], "_work": None, "_layer": None})

    def weights(self):
        """The packed weights the GEMM takes: resident, or expanded now from the resident 4-bit form."""
        if self.w_packed is not None:
            return self.w_packed
        return pack_weight_e3m2(self.qw, self.sw, out=_staging_buffer(packed_weight_e3m2_bytes(self.N, self.K), self.qw.device))

    def _workspace(self, M, device, layer):
        """The layer's buffers for M tokens, made again when anything that their sizes depend on has changed.  One object:
        a call takes all its buffers from the one that it got, whatever other threads do to the layer meanwhile.
        layer: what _descriptor(self.r) has just returned."""
        work = self._work
        if work is not None and work.layer is layer and work.y.shape[0] == M and work.y.device == device:
            return work
        key = (M, device, *layer.values[:4], self.w_packed is None)
        if work is not None and work.key == key:
            work = self._work = work._replace(layer=layer)
        else:
            lib, ref, K, r = load_library(), layer.address, self.K, self.r
            codes = torch.empty(act_e3m2_bytes(M, K) if self.container == "e3m2" else M * K // 2, dtype=torch.uint8, device=device)
            if self.container == "e3m2":
                qx, sx = ActE3M2(codes, M, K), None
            else:
                qx = codes.view(K // 64, M, 32)
                sx = (torch.empty((K // 64, M), dtype=torch.float32, device=device) if self.container == "nibble"
                      else torch.empty(((K // 64 + 1) // 2, M, 2, 2), dtype=torch.uint8, device=device))
            h = torch.empty((M, r), dtype=torch.float32, device=device) if r else None
            y = torch.empty((M, self.N), dtype=torch.bfloat16, device=device)
            n = lib.svdq_layer_scratch_bytes(ref, M)
            scratch = torch.empty(n, dtype=torch.uint8, device=device) if n else None
            # Room for expanded weights: the canonical form's is shared between layers (and reserved here, though few tokens
            # expand nothing).  The nibble container's is taken for each call: its layers may run on several streams at
            # once, and kept it would be as much again as the packed weights, in every layer.  So is the canonical form's where
            # svdq_layer_forward would do without.
            canonical = self.container == "e3m2" and self.w_packed is None
            staging, few = lib.svdq_layer_staging_bytes(ref, M), self.N >= 4096 and 2048 <= K <= 16384 and -(-M // 64) * -(-self.N // 64) <= 480
            shared = canonical and not few
            if canonical:
                _staging_buffer(packed_weight_e3m2_bytes(self.N, K), device)
            work = self._work = _Work(codes, sx, h, scratch, staging, shared, y, (qx, sx, h, y),
                                      tuple(map(_addr, (codes, sx, h, scratch))), y.data_ptr(), key, layer)
        return work

    def buffers(self, M, device):
        """(qx, sx, h, y) for M tokens: what quantize() fills and gemm() takes, and the output."""
        device = torch.device(device)
        if device.type == "cuda" and device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        return self._workspace(M, device, self._descriptor(self.r)).public

    def _staging(self, work, device):
        """Memory for one call's expanded operands, or None; the caller holds it until its kernels are enqueued."""
        if not work.staging:
            return None
        return (_staging_buffer(packed_weight_e3m2_bytes(self.N, self.K), device) if work.shared
                else torch.empty(work.staging, dtype=torch.uint8, device=device))

    def quantize(self, x_bf16, rho, gelu=False):
        """Kernel (a) into the layer's buffers; gelu=True applies the feed-forward block's activation on the fly."""
        out = self.buffers(x_bf16.shape[0], x_bf16.device)[:3]
        if gelu:
            return quantize_act_gelu(self.format, x_bf16, self.inv_lambda, rho, self.l1_packed, self.r, out=out)
        fn = {"e3m2": quantize_act_e3m2, "nibble": quantize_act, "mxfp4": quantize_act_mxfp4}[self.container]
        return fn(x_bf16, self.inv_lambda, rho, self.l1_packed, self.r, out=out)

    def gemm(self, qx, sx, h):
        codes = qx.buf if self.container == "e3m2" else qx
        M, device = (qx.M if self.container == "e3m2" else qx.shape[1]), codes.device
        work, layer = self._workspace(M, device, self._descriptor(self.r)), self._descriptor(0 if h is None else h.shape[1])
        staging = self._staging(work, device) if work.shared else None       # nibbles are multiplied as they are
        _check(load_library().svdq_layer_gemm(
            layer.address, codes.data_ptr(), _addr(sx), _addr(h), M, _addr(staging),
            work.y_ptr, self.N, _raw_stream()), "svdq_layer_gemm")
        return work.y

    def forward(self, x_bf16, rho, gelu=False):
        """The layer's output, in the layer's own buffer, which the next call writes again.  x may be that buffer."""
        M, K = x_bf16.shape
        # the MXFP4 pass also takes the bits in another two-byte type, as quantize_act_mxfp4 does
        assert x_bf16.dtype == torch.bfloat16 or (self.container == "mxfp4" and not gelu and x_bf16.element_size() == 2)
        assert x_bf16.stride(1) == 1 and K == self.K
        device = x_bf16.device
        layer = self._descriptor(self.r)
        work = self._workspace(M, device, layer)
        staging = self._staging(work, device) if work.staging else None
        _check((_lib or load_library()).svdq_layer_forward(
            layer.address, x_bf16.data_ptr(), x_bf16.stride(0) if M > 1 else K, float(rho), 1 if gelu else 0, M,
            *work.ptrs, None if staging is None else staging.data_ptr(),
            work.y_ptr, self.N, _raw_stream()), "svdq_layer_forward")
        return work.y


# ---- the 8-bit layer, and its form grouped by expert ---------------------------------------------
# Arguments are checked here for what the C functions cannot see (types, shapes, devices): a few comparisons a tensor, words only
# where one fails, since calls with few tokens wait for the host.
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_stream_of = getattr(torch._C, "_cuda_getCurrentRawStream", lambda gpu: torch.cuda.current_stream(gpu).cuda_stream)


def _gpu(t):
    """The GPU that holds t, which has to be the current one."""
    gpu = t.get_device()
    if gpu >= 0 and gpu == _current_device():
        return gpu
    raise ValueError(f"tensors on the current GPU are needed, not on {t.device}")


_BF16, _F32, _I8, _I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32


def _refuse(name, t, dtype, shape, gpu):
    wanted = " or ".join(map(str, dtype)) if isinstance(dtype, tuple) else dtype
    raise ValueError(f"{name}: {wanted} of shape {shape} is needed, rows of consecutive values, on GPU {gpu} (the current one); "
                     f"got {t.dtype} of shape {tuple(t.shape)}, strides {t.stride()}, on {t.device}")


def _vector(name, t, dtype, n, gpu):
    """A contiguous tensor of this type and n elements on GPU `gpu` -> its address."""
    if t.dtype is not dtype or t.numel() != n or t.get_device() != gpu or not t.is_contiguous():
        _refuse(name, t, dtype, f"[{n}]", gpu)
    return t.data_ptr()


def _tensor(name, t, dtype, shape, gpu):
    """The same with its shape."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != gpu or not t.is_contiguous():
        _refuse(name, t, dtype, shape, gpu)
    return t.data_ptr()


def _matrix(name, t, dtypes, gpu, cols=None):
    """A matrix on GPU `gpu` whose rows of consecutive values may be further apart than they are long -> (rows, columns, row stride)."""
    if t.dim() != 2 or t.dtype not in dtypes or t.get_device() != gpu:
        _refuse(name, t, dtypes, ("any", "any" if cols is None else cols), gpu)
    rows, n = t.shape
    ld, one = t.stride()
    if rows <= 1:
        ld = (n + 7) & ~7
    if (cols is not None and n != cols) or ld < n or (one != 1 and n > 1):
        _refuse(name, t, dtypes, (rows, n if cols is None else cols), gpu)
    return rows, n, ld


def _quantize_int8_out(out, M, K, x, gpu):
    if out is None:
        return torch.empty((M, K), dtype=_I8, device=x.device), torch.empty(M, dtype=_F32, device=x.device)
    _tensor("out[0]", out[0], _I8, (M, K), gpu)
    _vector("out[1]", out[1], _F32, M, gpu)
    return out


def quantize_act_int8(x_bf16, inv_lambda=None, rho=1.0, gelu=False, out=None):
    """x [M,K] bf16 (row stride allowed) -> (qx [M,K] int8, sx [M] f32): codes of x * inv_lambda (None: of x) with one scale
    (rho max|.|) / 127 a token; gelu=True: of gelu(x)."""
    gpu = _gpu(x_bf16)
    M, K, ldx = _matrix("x", x_bf16, (_BF16,), gpu)
    il = None if inv_lambda is None else _vector("inv_lambda", inv_lambda, _F32, K, gpu)
    qx, sx = _quantize_int8_out(out, M, K, x_bf16, gpu)
    if M:                            # an empty tensor has no address
        _check((_lib or load_library()).svdq_quantize_act_int8(x_bf16.data_ptr(), ldx, il, float(rho), 1 if gelu else 0, M, K, qx.data_ptr(), sx.data_ptr(),
                                                               _stream_of(gpu)), "svdq_quantize_act_int8")
    return qx, sx


def _linear_out(out, M, N, out_dtype, like, gpu):
    """(y, its row stride, its type's code)"""
    if out is None:
        if out_dtype is not _BF16 and out_dtype is not _F32:
            raise ValueError(f"out_dtype: bfloat16 or float32, not {out_dtype}")
        return torch.empty_strided((M, N), (N, 1), dtype=out_dtype, device=like.device), N, OUT_F32 if out_dtype is _F32 else OUT_BF16
    rows, _, ldy = _matrix("out", out, (_BF16, _F32), gpu, N)
    if rows != M:
        _refuse("out", out, (_BF16, _F32), (M, N), gpu)
    return out, ldy, OUT_F32 if out.dtype is _F32 else OUT_BF16


def linear_w8a8(qx, sx, qw, sw, bias=None, out=None, out_dtype=torch.bfloat16):
    """qx [M,K] int8, sx [M] f32, qw [N,K] int8, sw [N] f32, bias [N] f32 -> y [M,N] = (qx qw^T) sx sw + bias, bf16 or f32."""
    gpu = _gpu(qx)
    if qx.dim() != 2 or qw.dim() != 2:
        _refuse("qx, qw", qx if qx.dim() != 2 else qw, _I8, ("any", "any"), gpu)
    (M, K), N = qx.shape, qw.shape[0]
    pq, ps, pw, pc = _vector("qx", qx, _I8, M * K, gpu), _vector("sx", sx, _F32, M, gpu), _tensor("qw", qw, _I8, (N, K), gpu), _vector("sw", sw, _F32, N, gpu)
    pb = None if bias is None else _vector("bias", bias, _F32, N, gpu)
    y, ldy, code = _linear_out(out, M, N, out_dtype, qx, gpu)
    if M:
        _check((_lib or load_library()).svdq_linear_w8a8(pq, ps, pw, pc, pb, M, N, K, y.data_ptr(), ldy, code, _stream_of(gpu)), "svdq_linear_w8a8")
    return y


def _row_rho(rho, M, gpu):
    """(the ratio of all rows, or the address of every row's)"""
    if not torch.is_tensor(rho):
        return float(rho), None
    return 1.0, _vector("rho", rho, _F32, M, gpu)


def quantize_act_int8_grouped(x_bf16, offsets, inv_lambda=None, rho=1.0, rows=None, gelu=False, out=None):
    """quantize_act_int8 of rows in the experts' order: expert e owns rows offsets[e] .. offsets[e + 1] (int32 [E + 1]) and smooths them
    with inv_lambda[e] ([E,K]).  rows (int32 [M], any order, repeats allowed): row i is made of x[rows[i]]; None: of x[i].
    rho: a number or every row's ratio (f32 [M]).  Rows that no expert owns are not written."""
    gpu = _gpu(x_bf16)
    x_rows, K, ldx = _matrix("x", x_bf16, (_BF16,), gpu)
    M, E = (x_rows if rows is None else rows.numel()), offsets.numel() - 1
    o, r = _vector("offsets", offsets, _I32, E + 1, gpu), None if rows is None else _vector("rows", rows, _I32, M, gpu)
    il = None if inv_lambda is None else _tensor("inv_lambda", inv_lambda, _F32, (E, K), gpu)
    ratio, row_rho = _row_rho(rho, M, gpu)
    qx, sx = _quantize_int8_out(out, M, K, x_bf16, gpu)
    if M:
        _check((_lib or load_library()).svdq_quantize_act_int8_grouped(
            x_bf16.data_ptr(), ldx, x_rows, r, o, E, il, ratio, row_rho, 1 if gelu else 0, M, K, qx.data_ptr(), sx.data_ptr(), _stream_of(gpu)),
            "svdq_quantize_act_int8_grouped")
    return qx, sx


def linear_w8a8_grouped(qx, sx, offsets, qw, sw, bias=None, out=None, out_dtype=torch.bfloat16):
    """linear_w8a8 grouped by expert: rows offsets[e] .. offsets[e + 1] (int32 [E + 1]) of qx with qw[e] ([E,N,K] int8), sw[e] and bias[e]
    ([E,N] f32).  Rows that no expert owns are not written."""
    gpu = _gpu(qx)
    if qx.dim() != 2 or qw.dim() != 3:
        _refuse("qx, qw", qx if qx.dim() != 2 else qw, _I8, "[M, K], [E, N, K]", gpu)
    (M, K), (E, N, _) = qx.shape, qw.shape
    pq, ps, pw = _vector("qx", qx, _I8, M * K, gpu), _vector("sx", sx, _F32, M, gpu), _tensor("qw", qw, _I8, (E, N, K), gpu)
    pc, pb = _tensor("sw", sw, _F32, (E, N), gpu), None if bias is None else _tensor("bias", bias, _F32, (E, N), gpu)
    o = _vector("offsets", offsets, _I32, E + 1, gpu)
    y, ldy, code = _linear_out(out, M, N, out_dtype, qx, gpu)
    if M:
        _check((_lib or load_library()).svdq_linear_w8a8_grouped(pq, ps, pw, pc, pb, o, E, M, N, K, y.data_ptr(), ldy, code, _stream_of(gpu)), "svdq_linear_w8a8_grouped")
    return y


class _LayerInt8(ctypes.Structure):
    """svdq_layer_int8 of include/svdq.h."""
    _fields_ = [(n, _i32) for n in ("E", "N", "K")] + [(n, _vp) for n in ("inv_lambda", "qw", "sw", "bias")]


class _W8A8:
    """What W8A8Linear and W8A8Experts share.  The tensors are attributes and may be replaced; a call looks at what it finds."""

    def __init__(self, inv_lambda, qw, sw, bias=None):
        self.inv_lambda, self.qw, self.sw, self.bias = inv_lambda, qw, sw, bias
        self._held = None
        self._descriptor()

    def _descriptor(self):
        """svdq_layer_int8 of the tensors that the layer holds now, checked when they, or what a kernel goes by of them (memory, type, shape,
        order), have changed.  The caller keeps it through its call."""
        inv_lambda, qw, sw, bias = tensors = self.inv_lambda, self.qw, self.sw, self.bias
        held = self._held
        if held is not None:
            (a, b, c, d), (at, weights, channels, inputs), layer = held
            # (attributes only, 0.7 us of a call: making and comparing views costs more)
            if (a is inv_lambda and b is qw and c is sw and d is bias
                    and at == (None if a is None else a.data_ptr(), b.data_ptr(), c.data_ptr(), None if d is None else d.data_ptr())
                    and b.dtype is _I8 and c.dtype is _F32 and b.shape == weights and c.shape == channels and b.is_contiguous() and c.is_contiguous()
                    and (a is None or (a.dtype is _F32 and a.shape == inputs and a.is_contiguous()))
                    and (d is None or (d.dtype is _F32 and d.shape == channels and d.is_contiguous()))):
                return layer
        if qw.dim() != 2 + self.GROUPED:
            raise ValueError(f"qw: {'[E, N, K]' if self.GROUPED else '[N, K]'} is needed, not {tuple(qw.shape)}")
        lead, (N, K), gpu = tuple(qw.shape[:-2]), qw.shape[-2:], qw.get_device()
        weights, channels, inputs = lead + (N, K), lead + (N,), lead + (K,)
        at = (None if inv_lambda is None else _tensor("inv_lambda", inv_lambda, _F32, inputs, gpu), _tensor("qw", qw, _I8, weights, gpu),
              _tensor("sw", sw, _F32, channels, gpu), None if bias is None else _tensor("bias", bias, _F32, channels, gpu))
        layer = _LayerInt8(lead[0] if lead else 0, N, K, *at)
        layer.address, layer.shape = ctypes.addressof(layer), (layer.E, N, K, gpu)
        layer.rows_on_chip = (_lib or load_library()).svdq_layer_int8_rows_on_chip(layer.address)
        self._held = (tensors, (at, weights, channels, inputs), layer)
        return layer

    def __getstate__(self):
        """Copies make a descriptor of their own."""
        return {**self.__dict__, "_held": None}

    def _forward(self, x, layer, gpu, rows, offsets, rho, row_rho, gelu, M, out):
        """M: None for the rows of x."""
        _, N, K, home = layer.shape
        x_rows, _, ldx = _matrix("x", x, (_BF16,), gpu, K)
        if home != gpu:
            raise ValueError(f"x is on GPU {gpu}, the layer on {self.qw.device}")
        if M is None:
            M = x_rows
        if out is None:
            y, ldy = x.new_empty(M, N), N
        else:
            y, ldy, code = _linear_out(out, M, N, _BF16, x, gpu)
            if code != OUT_BF16:
                _refuse("out", out, _BF16, (M, N), gpu)
        if M:
            codes = scales = None
            if out is not None or M > layer.rows_on_chip:
                # of this call alone, from torch's allocator: calls on other streams and captured ones have their own
                work = x.new_empty(M * (K // 2 + 2))
                codes = work.data_ptr()
                scales = codes + M * K
            rc = (_lib or load_library()).svdq_layer_int8_forward(
                layer.address, x.data_ptr(), ldx, x_rows, rows, offsets, rho, row_rho, 1 if gelu else 0, M,
                codes, scales, y.data_ptr(), ldy, _stream_of(gpu))
            if rc:
                _check(rc, "svdq_layer_int8_forward")
        return y


class W8A8Linear(_W8A8):
    """One linear in 8 bits: qw [N,K] int8, sw [N] f32 (weight n is qw[n] sw[n]), bias [N] f32 or None, and the smoothing vector inv_lambda [K]
    f32 of its input, or None.  Holds references, lays nothing out, keeps no buffers: its calls may run on any streams at once."""
    GROUPED = 0

    def forward(self, x_bf16, rho=1.0, gelu=False, out=None):
        """x [M,K] bf16 -> y [M,N] bf16: quantize_act_int8 and linear_w8a8 in one call.  out may share memory with x."""
        return self._forward(x_bf16, self._descriptor(), _gpu(x_bf16), None, None, float(rho), None, gelu, None, out)


class W8A8Experts(_W8A8):
    """The linears of E experts: qw [E,N,K] int8, sw [E,N], bias [E,N] or None, inv_lambda [E,K] or None (f32)."""
    GROUPED = 1

    def forward(self, x_bf16, offsets, rho=1.0, rows=None, gelu=False, out=None):
        """y [M,N] bf16 in the experts' order: rows offsets[e] .. offsets[e + 1] are expert e's, made of x[rows] (rows int32 [M]) or of x;
        rho a number or every row's ratio (f32 [M]).  quantize_act_int8_grouped and linear_w8a8_grouped in one call; rows that no
        expert owns are not written (without `out`: hold anything)."""
        layer, gpu = self._descriptor(), _gpu(x_bf16)
        M = x_bf16.shape[0] if rows is None else rows.numel()
        o, r = _vector("offsets", offsets, _I32, layer.shape[0] + 1, gpu), None if rows is None else _vector("rows", rows, _I32, M, gpu)
        ratio, row_rho = _row_rho(rho, M, gpu)
        return self._forward(x_bf16, layer, gpu, r, o, ratio, row_rho, gelu, M, out)
