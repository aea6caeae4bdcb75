"""ctypes binding of libmxnorm.so (declared in include/mxnorm.h).

Argument marshalling only: each function checks tensor dtypes, devices and
shapes, allocates outputs with ``torch.empty`` when none are given, and calls
the C entry point of the same name on the current HIP stream.  Every step of
the computation runs in the library's HIP kernels.  There is no fallback: if
the library is missing, or a tensor is not on the GPU, a call raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxnorm.so")

MX_OK, MX_EINVAL, MX_EUNSUPPORTED, MX_EHIP = 0, 1, 2, 3
SCALE_MODES = {"rceil": 0, "floor": 1}
OUT_DTYPES = {torch.float32: 0, torch.bfloat16: 1}
ELEMS = {"e4m3": 0, "e2m1": 1}
ACTS = {"silu": 0, "gelu_tanh": 1}
# the gated product's outputs; torch.uint8 stands for MX codes with their scales
GATED_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.uint8: 2}
ABI_VERSION = 1
MAX_D = 32768

_lib = None


class MXNormError(RuntimeError):
    def __init__(self, status, detail):
        super().__init__("%s (%s)" % (detail, _status_name(status)))
        self.status = status


def _status_name(status):
    return {0: "MX_OK", 1: "MX_EINVAL", 2: "MX_EUNSUPPORTED", 3: "MX_EHIP"}.get(status, str(status))


def load():
    """Load libmxnorm.so and declare its signatures (no GPU work)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libmxnorm.so is not built (expected at %s); run "
                           "__graft_entry__.build()" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    P, I64, I, F = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int, ctypes.c_float
    sigs = {
        "mxnorm_mxfp8_fwd": (I, [P, I64, I64, I, F, F, I, P, P, P, P]),
        "rmsnorm_mxfp8_fwd": (I, [P, P, I64, I64, F, I, P, P, P, P]),
        "mxnorm_nvfp4_fwd": (I, [P, I64, I64, I, F, F, F, P, P, P, P]),
        "rmsnorm_nvfp4_fwd": (I, [P, P, I64, I64, F, F, P, P, P, P]),
        "mxnorm_mx_fwd": (I, [P, I64, I64, I, I, I, F, F, I, P, P, P, P]),
        "rmsnorm_mx_fwd": (I, [P, P, I64, I64, I, I, F, I, P, P, P, P]),
        "mxnorm_postround_mx_fwd": (I, [P, I64, I64, I, I, F, I, P, P, P, P]),
        "mxnorm_postround_table": (I, [I, P, P]),
        "mx_cast_fwd": (I, [P, P, I64, I64, I, I, I, P, P, P]),
        "mx_matmul_fwd": (I, [P, P, P, P, I64, I64, I64, I, I, P, I, P, P]),
        "mx_cast_t_fwd": (I, [P, P, I64, I64, I, I, I, P, P, P]),
        "mxnorm_ste_bwd_workspace_bytes": (ctypes.c_size_t, [I64, I64]),
        "mxnorm_ste_bwd": (I, [P, P, P, P, I64, I64, I, P, P, P, ctypes.c_size_t, P]),
        "mxnorm_ste_bwd_noalloc_max_workspace": (ctypes.c_size_t, []),
        "mxnorm_ste_bwd_noalloc": (I, [P, P, P, P, I64, I64, I, P, P, P]),
        "mxnorm_linear_fwd_workspace_bytes": (ctypes.c_size_t, [I64, I64, I, I]),
        "mxnorm_linear_fwd": (I, [P, I64, I64, P, P, I64, I, I, I, F, F, I, I, P, P, P,
                                  ctypes.c_size_t, P]),
        "mx_gated_fwd": (I, [P, P, P, P, I64, I64, I64, I, I, I, I, I, P, P, P, P]),
        "mxnorm_gated_fwd_workspace_bytes": (ctypes.c_size_t, [I64, I64, I, I]),
        "mxnorm_gated_fwd": (I, [P, I64, I64, P, P, I64, I, I, I, F, F, I, I, I, P, P, P, P, P,
                                 ctypes.c_size_t, P]),
        "mx_gated_bwd": (I, [P, P, I64, I64, I, P, P]),
        "mxnorm_gated_bwd_workspace_bytes": (ctypes.c_size_t, [I64, I64, I64, I]),
        "mxnorm_gated_bwd": (I, [P, P, P, P, P, P, I64, I64, I64, I, I, I, I, I, P, P, P, P,
                                 ctypes.c_size_t, P]),
        "mxnorm_linear_bwd_workspace_bytes": (ctypes.c_size_t, [I64, I64, I64, I]),
        "mxnorm_linear_bwd": (I, [P, P, P, P, P, I64, I64, I64, I, I, I, P, P, P, P,
                                  ctypes.c_size_t, P]),
        "qk_norm_rope_fwd": (I, [P, P, P, P, I64, I64, I64, P, P, I, F, P, P, P]),
        "qk_norm_rope_bwd_workspace_bytes": (ctypes.c_size_t, [I64, I64]),
        "qk_norm_rope_bwd": (I, [P, P, P, P, P, P, I64, I64, I64, P, P, I, F, P, P, P, P, P,
                                 ctypes.c_size_t, P]),
        "window_attn_fwd": (I, [P, P, P, I64, I64, I64, P, P, I64, I64, I64, F, P, P, P]),
        "window_attn_bwd_workspace_bytes": (ctypes.c_size_t, [I64] * 8),
        "window_attn_bwd": (I, [P, P, P, P, P, P, I64, I64, I64, P, P, I64, I64, I64, F, P, P, P, P,
                                ctypes.c_size_t, P]),
        "kv_cache_append": (I, [P, P, P, I64, I64, I64, P, I64, P, P, I64, P, P]),
        "kv_cache_attn_fwd_workspace_bytes": (ctypes.c_size_t, [I64] * 11),
        "kv_cache_attn_fwd": (I, [P, P, I64, I64, P, I64, P, P, I64, I64, I64, P, I64, I64, F, P, P,
                                  ctypes.c_size_t, P]),
        "mxnorm_default_global_scale": (F, [I64, I, I, F]),
        "rmsnorm_default_global_scale": (F, [I64, F]),
        "mxnorm_coef": (F, [I, I]),
        "mx_status_str": (ctypes.c_char_p, [I]),
        "mx_last_error": (ctypes.c_char_p, []),
        "mxnorm_abi_version": (I, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    if lib.mxnorm_abi_version() != ABI_VERSION:
        raise RuntimeError("libmxnorm.so ABI version %d, binding expects %d"
                           % (lib.mxnorm_abi_version(), ABI_VERSION))
    _lib = lib
    return lib


def _check(status):
    if status != MX_OK:
        raise MXNormError(status, load().mx_last_error().decode() or "error")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(device):
    # the handle of torch.cuda.current_stream(device), without building the
    # Stream object around it (1.5 us a call)
    return torch._C._cuda_getCurrentRawStream(device.index)


def _input(x):
    if not isinstance(x, torch.Tensor) or x.dtype != torch.bfloat16 or x.dim() != 2:
        raise TypeError("x must be a 2-D torch.bfloat16 tensor [T, d]")
    if not x.is_cuda:
        raise RuntimeError("x must be on the GPU: libmxnorm has no CPU path")
    if not x.is_contiguous():
        raise ValueError("x must be contiguous")
    return x.shape[0], x.shape[1]


def _gamma(gamma, x):
    if gamma is None:
        return None
    if gamma.dtype != torch.bfloat16 or gamma.shape != (x.shape[1],) or gamma.device != x.device:
        raise TypeError("gamma must be a bfloat16 [d] tensor on x's device")
    return gamma.contiguous()


def _out(t, shape, dtype, device):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError("output tensor must be contiguous %s %s on %s" % (dtype, shape, device))
    return t


def mxnorm_mxfp8_fwd(x, p=2, coef=0.0, eps=1e-6, scale_mode="rceil",
                     codes=None, scales=None, rho=None, want_rho=True):
    """MXNorm (Algorithm 2) with MXFP8 output.

    Returns (codes uint8 [T, d] E4M3, scales uint8 [T, d/32] E8M0,
    rho float32 [T] or None)."""
    T, d = _input(x)
    codes = _out(codes, (T, d), torch.uint8, x.device)
    scales = _out(scales, (T, d // 32), torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().mxnorm_mxfp8_fwd(_ptr(x), T, d, p, coef, eps, SCALE_MODES[scale_mode],
                                   _ptr(codes), _ptr(scales), _ptr(rho) if want_rho else None,
                                   _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def rmsnorm_mxfp8_fwd(x, gamma=None, eps=1e-6, scale_mode="rceil",
                      codes=None, scales=None, rho=None, want_rho=True):
    """RMSNorm (+ optional gain) then MXFP8 cast (Algorithm 1)."""
    T, d = _input(x)
    g = _gamma(gamma, x)
    codes = _out(codes, (T, d), torch.uint8, x.device)
    scales = _out(scales, (T, d // 32), torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().rmsnorm_mxfp8_fwd(_ptr(x), _ptr(g), T, d, eps, SCALE_MODES[scale_mode],
                                    _ptr(codes), _ptr(scales), _ptr(rho) if want_rho else None,
                                    _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def mxnorm_nvfp4_fwd(x, global_scale=None, p=2, coef=0.0, eps=1e-6,
                     codes=None, scales=None, rho=None, want_rho=True):
    """MXNorm with NVFP4 output.  global_scale None selects the Lemma-2
    default.  Returns (packed E2M1 codes uint8 [T, d/2], E4M3 scales uint8
    [T, d/16], rho)."""
    T, d = _input(x)
    if global_scale is None:
        global_scale = mxnorm_default_global_scale(d, 16, p, coef)
    codes = _out(codes, (T, d // 2), torch.uint8, x.device)
    scales = _out(scales, (T, d // 16), torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().mxnorm_nvfp4_fwd(_ptr(x), T, d, p, coef, eps, global_scale, _ptr(codes),
                                   _ptr(scales), _ptr(rho) if want_rho else None,
                                   _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def rmsnorm_nvfp4_fwd(x, gamma=None, global_scale=None, eps=1e-6,
                      codes=None, scales=None, rho=None, want_rho=True):
    T, d = _input(x)
    g = _gamma(gamma, x)
    if global_scale is None:
        if g is not None:
            raise ValueError("pass global_scale when gamma is given; "
                             "rmsnorm_default_global_scale(d, max|gamma|) is the Lemma-1 default")
        global_scale = rmsnorm_default_global_scale(d, 1.0)
    codes = _out(codes, (T, d // 2), torch.uint8, x.device)
    scales = _out(scales, (T, d // 16), torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().rmsnorm_nvfp4_fwd(_ptr(x), _ptr(g), T, d, eps, global_scale, _ptr(codes),
                                    _ptr(scales), _ptr(rho) if want_rho else None,
                                    _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def _mx_out_shapes(T, d, block, elem):
    if block not in (16, 32, 64) or elem not in ELEMS:
        raise ValueError("block must be 16, 32 or 64 and elem 'e4m3' or 'e2m1'")
    return ((T, d) if elem == "e4m3" else (T, d // 2)), (T, d // block)


def mxnorm_mx_fwd(x, block=32, elem="e4m3", p=2, coef=0.0, eps=1e-6, scale_mode="rceil",
                  codes=None, scales=None, rho=None, want_rho=True):
    """MXNorm with a general MX output: E8M0 scales per `block` elements and
    E4M3 or E2M1 (packed two per byte) codes."""
    T, d = _input(x)
    cs, ss = _mx_out_shapes(T, d, block, elem)
    codes = _out(codes, cs, torch.uint8, x.device)
    scales = _out(scales, ss, torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().mxnorm_mx_fwd(_ptr(x), T, d, block, ELEMS[elem], p, coef, eps,
                                SCALE_MODES[scale_mode], _ptr(codes), _ptr(scales),
                                _ptr(rho) if want_rho else None, _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def mxnorm_postround_mx_fwd(x, block=32, elem="e4m3", eps=1e-6, scale_mode="rceil",
                            codes=None, scales=None, rho=None, want_rho=True):
    """Post-round MXNorm (the post-round appendix): rho~ from the block
    absmaxes rounded down to powers of two, through the inverse of
    f(sigma) = E[max r(|X|)], then the MX cast of Algorithm 2."""
    T, d = _input(x)
    cs, ss = _mx_out_shapes(T, d, block, elem)
    codes = _out(codes, cs, torch.uint8, x.device)
    scales = _out(scales, ss, torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().mxnorm_postround_mx_fwd(_ptr(x), T, d, block, ELEMS[elem], eps,
                                          SCALE_MODES[scale_mode], _ptr(codes), _ptr(scales),
                                          _ptr(rho) if want_rho else None, _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def mxnorm_postround_table(block):
    """The library's post-round table: (x, v) float32 arrays of 65 points."""
    import numpy as np
    xs = np.empty(65, np.float32)
    vs = np.empty(65, np.float32)
    _check(load().mxnorm_postround_table(block, xs.ctypes.data_as(ctypes.c_void_p),
                                         vs.ctypes.data_as(ctypes.c_void_p)))
    return xs, vs


def rmsnorm_mx_fwd(x, gamma=None, block=32, elem="e4m3", eps=1e-6, scale_mode="rceil",
                   codes=None, scales=None, rho=None, want_rho=True):
    """RMSNorm (+ optional gain) then the general MX cast."""
    T, d = _input(x)
    g = _gamma(gamma, x)
    cs, ss = _mx_out_shapes(T, d, block, elem)
    codes = _out(codes, cs, torch.uint8, x.device)
    scales = _out(scales, ss, torch.uint8, x.device)
    if want_rho:
        rho = _out(rho, (T,), torch.float32, x.device)
    _check(load().rmsnorm_mx_fwd(_ptr(x), _ptr(g), T, d, block, ELEMS[elem], eps,
                                 SCALE_MODES[scale_mode], _ptr(codes), _ptr(scales),
                                 _ptr(rho) if want_rho else None, _stream(x.device)))
    return codes, scales, (rho if want_rho else None)


def mx_cast_fwd(x, gamma=None, block=32, elem="e4m3", scale_mode="rceil",
                codes=None, scales=None):
    """Plain MX cast of x (or RN(x * gamma)), no normalisation.  With x a
    weight [N, d] and gamma the norm gain this is the gain-folded weight cast
    of the MXNormLinear forward (Sec. 3.7)."""
    T, d = _input(x)
    g = _gamma(gamma, x)
    cs, ss = _mx_out_shapes(T, d, block, elem)
    codes = _out(codes, cs, torch.uint8, x.device)
    scales = _out(scales, ss, torch.uint8, x.device)
    _check(load().mx_cast_fwd(_ptr(x), _ptr(g), T, d, block, ELEMS[elem],
                              SCALE_MODES[scale_mode], _ptr(codes), _ptr(scales),
                              _stream(x.device)))
    return codes, scales


def _mx_operand(codes, scales, K, block, elem, name):
    cw = K if elem == "e4m3" else K // 2
    for t, shape_ok in ((codes, codes.dim() == 2 and codes.shape[1] == cw),
                        (scales, scales.dim() == 2 and scales.shape[1] == K // block)):
        if t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous() or not shape_ok:
            raise ValueError("%s: codes must be contiguous uint8 [rows, %d] and scales [rows, %d] "
                             "on the GPU" % (name, cw, K // block))
    if codes.shape[0] != scales.shape[0]:
        raise ValueError("%s: codes and scales disagree on the row count" % name)
    return codes.shape[0]


def mx_matmul_fwd(a_codes, a_scales, b_codes, b_scales, K, block=32, elem="e4m3",
                  out_dtype=torch.float32, out=None, b_gain=None):
    """H = dec(A) dec(B)^T on the block-scaled matrix cores (Sec. 3.7 eq.
    (mx-matmul)).  A: MX codes/scales [M, .] along K; B: [N, .].  b_gain
    (bf16 [N]) multiplies column n of H after the product.  Returns H [M, N]
    in out_dtype (float32 or bfloat16).  The order of the float additions, and
    with it a row's last bits, may depend on M, N and K."""
    if elem not in ELEMS or out_dtype not in OUT_DTYPES:
        raise ValueError("elem must be 'e4m3' or 'e2m1', out_dtype float32 or bfloat16")
    M = _mx_operand(a_codes, a_scales, K, block, elem, "A")
    N = _mx_operand(b_codes, b_scales, K, block, elem, "B")
    if b_gain is not None and (b_gain.dtype != torch.bfloat16 or b_gain.shape != (N,) or
                               b_gain.device != a_codes.device or not b_gain.is_contiguous()):
        raise ValueError("b_gain must be a contiguous bfloat16 [N] tensor on the GPU")
    out = _out(out, (M, N), out_dtype, a_codes.device)
    _check(load().mx_matmul_fwd(_ptr(a_codes), _ptr(a_scales), _ptr(b_codes), _ptr(b_scales),
                                M, N, K, block, ELEMS[elem], _ptr(b_gain),
                                OUT_DTYPES[out_dtype], _ptr(out), _stream(a_codes.device)))
    return out


def mxnorm_linear_fwd(x, w_codes, w_scales, block=32, elem="e4m3", p=2, coef=0.0, eps=1e-6,
                      scale_mode="rceil", out_dtype=torch.bfloat16):
    """The MXNormLinear forward H = MXNorm(X) MXCast(W gamma)^T (Sec. 3.7):
    MXNorm of the activations, then the MX matmul with a weight cast once by
    mx_cast_fwd(W, gamma).  Returns (H, rho~)."""
    T, d = _input(x)
    _mx_out_shapes(T, d, block, elem)
    mode = SCALE_MODES[scale_mode]
    if out_dtype not in OUT_DTYPES:
        raise ValueError("elem must be 'e4m3' or 'e2m1', out_dtype float32 or bfloat16")
    N = _mx_operand(w_codes, w_scales, d, block, elem, "B")
    lib, e = load(), ELEMS[elem]
    h = torch.empty((T, N), dtype=out_dtype, device=x.device)
    rho = torch.empty((T,), dtype=torch.float32, device=x.device)
    ws_bytes = lib.mxnorm_linear_fwd_workspace_bytes(T, d, block, e)
    ws = torch.empty((ws_bytes,), dtype=torch.uint8, device=x.device)
    _check(lib.mxnorm_linear_fwd(x.data_ptr(), T, d, w_codes.data_ptr(), w_scales.data_ptr(), N,
                                 block, e, p, coef, eps, mode, OUT_DTYPES[out_dtype],
                                 h.data_ptr(), rho.data_ptr(), ws.data_ptr(), ws_bytes,
                                 _stream(x.device)))
    return h, rho


def _call(fn, device, *args):
    """fn(*args, stream) with `device` current: a stream handle of 0 is the
    current device's default stream."""
    if torch._C._cuda_getDevice() == device.index:
        status = fn(*args, _stream(device))
    else:
        with torch.cuda.device(device):
            status = fn(*args, _stream(device))
    _check(status)


def _gated_outputs(T, F, elem, act, out_dtype, save_gu, a):
    """(out, scales or None, gu or None) of a gated product of a.  (new_empty:
    0.5 us a tensor less than empty with a device.)"""
    if elem not in ELEMS or act not in ACTS:
        raise ValueError("elem must be 'e4m3' or 'e2m1', act 'silu' or 'gelu_tanh'")
    if out_dtype not in GATED_DTYPES:
        raise ValueError("out_dtype must be float32, bfloat16 or uint8 (MX codes)")
    if out_dtype is torch.uint8:
        out = a.new_empty((T, F if elem == "e4m3" else F // 2), dtype=torch.uint8)
        scales = a.new_empty((T, F // 32), dtype=torch.uint8)
    else:
        out = a.new_empty((T, F), dtype=out_dtype)
        scales = None
    gu = a.new_empty((T, 2 * F), dtype=torch.bfloat16) if save_gu else None
    return out, scales, gu


def _gated_weight(w_codes, w_scales, K, block, elem, device):
    """F of a gate and up weight [2F, K]."""
    if elem not in ELEMS:
        raise ValueError("elem must be 'e4m3' or 'e2m1'")
    rows = _mx_operand(w_codes, w_scales, K, block, elem, "W")
    if rows % 2 or w_codes.device != device or w_scales.device != device:
        raise ValueError("W must have F gate rows and then F up rows, on the activations' device")
    return rows // 2


def mx_gated_fwd(a_codes, a_scales, w_codes, w_scales, K, block=32, elem="e4m3", act="silu",
                 out_dtype=torch.bfloat16, scale_mode="rceil", save_gu=False):
    """H = act(G) U with G and U the products of A [M, .] with the F gate and
    the F up rows of W [2F, .], both MX codes and scales along K, in one kernel.
    act: "silu" or "gelu_tanh".  out_dtype: float32, bfloat16, or uint8 for the
    MX encoding of H along F in `elem`.  Returns (H, gu): H [M, F], or (codes,
    scales) for uint8; gu bfloat16 [M, 2F], what the backward takes, or None."""
    F = _gated_weight(w_codes, w_scales, K, block, elem, a_codes.device)
    M = _mx_operand(a_codes, a_scales, K, block, elem, "A")
    if a_scales.device != a_codes.device:
        raise ValueError("A: codes and scales must be on one device")
    mode = SCALE_MODES[scale_mode]
    out, scales, gu = _gated_outputs(M, F, elem, act, out_dtype, save_gu, a_codes)
    _call(load().mx_gated_fwd, a_codes.device, a_codes.data_ptr(), a_scales.data_ptr(),
          w_codes.data_ptr(), w_scales.data_ptr(), M, F, K, block, ELEMS[elem], ACTS[act], mode,
          GATED_DTYPES[out_dtype], out.data_ptr(), _ptr(scales), _ptr(gu))
    return (out if scales is None else (out, scales)), gu


def mxnorm_gated_fwd(x, w_codes, w_scales, block=32, elem="e4m3", p=2, coef=0.0, eps=1e-6,
                     scale_mode="rceil", act="silu", out_dtype=torch.bfloat16, save_gu=False,
                     want_rho=True):
    """The gated feed-forward's first half: MXNorm of the activations x bf16
    [T, d], then mx_gated_fwd with a weight [2F, d] cast once by mx_cast_fwd(W,
    gamma).  Returns (H, gu, rho~) with H and gu as mx_gated_fwd's and rho~
    float32 [T] or None.  With out_dtype=torch.uint8 the down projection is
    mx_matmul_fwd(*H, down_codes, down_scales, F)."""
    T, d = _input(x)
    _mx_out_shapes(T, d, block, elem)
    F = _gated_weight(w_codes, w_scales, d, block, elem, x.device)
    mode = SCALE_MODES[scale_mode]
    out, scales, gu = _gated_outputs(T, F, elem, act, out_dtype, save_gu, x)
    rho = x.new_empty((T,), dtype=torch.float32) if want_rho else None
    lib, e = load(), ELEMS[elem]
    ws_bytes = lib.mxnorm_gated_fwd_workspace_bytes(T, d, block, e)
    ws = x.new_empty((ws_bytes,), dtype=torch.uint8)
    _call(lib.mxnorm_gated_fwd, x.device, x.data_ptr(), T, d, w_codes.data_ptr(),
          w_scales.data_ptr(), F, block, e, p, coef, eps, mode, ACTS[act], GATED_DTYPES[out_dtype],
          out.data_ptr(), _ptr(scales), _ptr(gu), _ptr(rho), ws.data_ptr(), ws_bytes)
    return (out if scales is None else (out, scales)), gu, rho


def _gated_gradient(grad_h, gu, act):
    """(T, F) of a gated product's gradient and kept products."""
    T, F = _input(grad_h)
    _input(gu)
    if gu.shape != (T, 2 * F) or gu.device != grad_h.device:
        raise ValueError("gu must be [T, 2F] for a grad_h [T, F], on its device")
    if act not in ACTS:
        raise ValueError("act must be 'silu' or 'gelu_tanh'")
    return T, F


def mx_gated_bwd(grad_h, gu, act="silu", grad_gu=None):
    """The gradient of both projections of mx_gated_fwd: bfloat16 [T, 2F] (gate
    columns, then up columns) from grad_h bfloat16 [T, F] and the forward's gu
    [T, 2F], which grad_gu may be."""
    T, F = _gated_gradient(grad_h, gu, act)
    grad_gu = _out(grad_gu, (T, 2 * F), torch.bfloat16, grad_h.device)
    _call(load().mx_gated_bwd, grad_h.device, grad_h.data_ptr(), gu.data_ptr(), T, F, ACTS[act],
          grad_gu.data_ptr())
    return grad_gu


def mxnorm_gated_bwd(grad_h, gu, x, rho, gamma, w, block=32, elem="e4m3", act="silu",
                     grad_x_dtype=torch.bfloat16, grad_dtype=torch.float32):
    """The backward of mxnorm_gated_fwd, every product and cast in the library,
    for any number of tokens:
      grad_P = mx_gated_bwd(grad_h, gu)                 [T, 2F]
      grad_Z = MXCast(grad_P) MXCast_2F(W)
      grad_X, grad_gamma = STE(X, grad_Z, gamma, rho~)
      grad_W = (MXCast(grad_P^T) MXCast(rho~ X)^T) . gamma
    grad_h bf16 [T, F]; gu bf16 [T, 2F] and rho float32 [T] from the forward; x
    bf16 [T, d]; gamma bf16 [d] or None; w bf16 [2F, d], before its cast.
    Returns (grad_x, grad_gamma [d], grad_w [2F, d]), the last two in
    grad_dtype (float32 or bfloat16)."""
    T, F = _gated_gradient(grad_h, gu, act)
    if _input(x)[0] != T:
        raise ValueError("x must have grad_h's rows")
    d = x.shape[1]
    _input(w)
    if w.shape != (2 * F, d):
        raise ValueError("w must be [2F, d]")
    if block not in (16, 32, 64) or elem not in ELEMS:
        raise ValueError("block must be 16, 32 or 64 and elem 'e4m3' or 'e2m1'")
    if x.device != grad_h.device or w.device != grad_h.device:
        raise ValueError("grad_h, x and w must be on one device")
    if rho.dtype != torch.float32 or rho.shape != (T,) or rho.device != x.device \
            or not rho.is_contiguous():
        raise ValueError("rho must be a contiguous float32 [T] tensor on x's device")
    if gamma is not None:
        _gamma(gamma, x)
        if not gamma.is_contiguous():
            raise ValueError("gamma must be contiguous")
    if grad_x_dtype not in OUT_DTYPES or grad_dtype not in OUT_DTYPES:
        raise ValueError("grad_x_dtype and grad_dtype must be float32 or bfloat16")
    lib, e = load(), ELEMS[elem]
    grad_x = x.new_empty((T, d), dtype=grad_x_dtype)
    grad_gamma = x.new_empty((d,), dtype=grad_dtype)
    grad_w = x.new_empty((2 * F, d), dtype=grad_dtype)
    ws_bytes = lib.mxnorm_gated_bwd_workspace_bytes(T, F, d, e)
    ws = x.new_empty((ws_bytes,), dtype=torch.uint8)
    _call(lib.mxnorm_gated_bwd, x.device, grad_h.data_ptr(), gu.data_ptr(), x.data_ptr(),
          rho.data_ptr(), _ptr(gamma), w.data_ptr(), T, F, d, block, e, ACTS[act],
          OUT_DTYPES[grad_x_dtype], OUT_DTYPES[grad_dtype], grad_x.data_ptr(), grad_gamma.data_ptr(),
          grad_w.data_ptr(), ws.data_ptr(), ws_bytes)
    return grad_x, grad_gamma, grad_w


def mx_cast_t_fwd(x, rho=None, block=32, elem="e4m3", scale_mode="rceil", codes=None,
                  scales=None):
    """Column-wise MX cast (Sec. 3.7): the MX encoding of (rho[:, None] * x)^T,
    blocked along x's rows.  x bf16 [R, C] -> codes [C, R] (E4M3) or
    [C, R/2] (E2M1), scales [C, R/32]."""
    R, C = _input(x)
    if rho is not None and (rho.dtype != torch.float32 or rho.shape != (R,) or
                            rho.device != x.device or not rho.is_contiguous()):
        raise ValueError("rho must be a contiguous float32 [R] tensor on x's device")
    if elem not in ELEMS:
        raise ValueError("elem must be 'e4m3' or 'e2m1'")
    codes = _out(codes, (C, R) if elem == "e4m3" else (C, R // 2), torch.uint8, x.device)
    scales = _out(scales, (C, R // block), torch.uint8, x.device)
    _check(load().mx_cast_t_fwd(_ptr(x), _ptr(rho), R, C, block, ELEMS[elem],
                                SCALE_MODES[scale_mode], _ptr(codes), _ptr(scales),
                                _stream(x.device)))
    return codes, scales


def mxnorm_ste_bwd(x, grad_z, gamma, rho, out_dtype=torch.bfloat16, want_grad_gamma=True,
                   grad_x=None, grad_gamma=None, workspace=None):
    """The straight-through estimator of the MXNorm backward (Sec. 3.7; the
    RMSNorm-gradient appendix with S = 1/rho~).  x, grad_z bf16 [T, d];
    gamma bf16 [d] or None; rho float32 [T] from the forward.  Returns
    (grad_x [T, d] in out_dtype, grad_gamma float32 [d] or None)."""
    T, d = _input(x)
    if grad_z.dtype != torch.bfloat16 or grad_z.shape != x.shape or grad_z.device != x.device \
            or not grad_z.is_contiguous():
        raise ValueError("grad_z must be a contiguous bfloat16 tensor shaped like x")
    g = _gamma(gamma, x)
    if rho.dtype != torch.float32 or rho.shape != (T,) or rho.device != x.device:
        raise ValueError("rho must be float32 [T] on x's device")
    if out_dtype not in OUT_DTYPES:
        raise ValueError("out_dtype must be float32 or bfloat16")
    lib = load()
    grad_x = _out(grad_x, (T, d), out_dtype, x.device)
    ws_bytes = 0
    if want_grad_gamma:
        grad_gamma = _out(grad_gamma, (d,), torch.float32, x.device)
        ws_bytes = int(lib.mxnorm_ste_bwd_workspace_bytes(T, d))
        if workspace is None:
            workspace = torch.empty(max(ws_bytes, 16), dtype=torch.uint8, device=x.device)
        elif workspace.numel() * workspace.element_size() < ws_bytes:
            raise ValueError("workspace smaller than mxnorm_ste_bwd_workspace_bytes(T, d)")
        ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.mxnorm_ste_bwd(_ptr(x), _ptr(grad_z), _ptr(g), _ptr(rho.contiguous()), T, d,
                              OUT_DTYPES[out_dtype], _ptr(grad_x),
                              _ptr(grad_gamma) if want_grad_gamma else None,
                              _ptr(workspace) if want_grad_gamma else None, ws_bytes,
                              _stream(x.device)))
    return grad_x, (grad_gamma if want_grad_gamma else None)


def mxnorm_ste_bwd_noalloc(x, grad_z, gamma, rho, grad_x, grad_gamma=None):
    """mxnorm_ste_bwd through the library's allocation-free entry point: the
    grad_gamma workspace is the library's static device array, so neither the
    library nor this call allocates.  The caller passes the outputs: grad_x
    [T, d] (float32 or bfloat16, its dtype selects the output type) and
    grad_gamma float32 [d] or None.  Calls that overlap in time on one GPU
    share that array and race."""
    T, d = _input(x)
    if grad_z.dtype != torch.bfloat16 or grad_z.shape != x.shape or grad_z.device != x.device \
            or not grad_z.is_contiguous():
        raise ValueError("grad_z must be a contiguous bfloat16 tensor shaped like x")
    g = _gamma(gamma, x)
    if rho.dtype != torch.float32 or rho.shape != (T,) or rho.device != x.device \
            or not rho.is_contiguous():
        raise ValueError("rho must be contiguous float32 [T] on x's device")
    if grad_x.dtype not in OUT_DTYPES or grad_x.shape != x.shape or grad_x.device != x.device \
            or not grad_x.is_contiguous():
        raise ValueError("grad_x must be a contiguous float32 or bfloat16 tensor shaped like x")
    if grad_gamma is not None and (grad_gamma.dtype != torch.float32 or grad_gamma.shape != (d,)
                                   or grad_gamma.device != x.device):
        raise ValueError("grad_gamma must be float32 [d] on x's device")
    _check(load().mxnorm_ste_bwd_noalloc(_ptr(x), _ptr(grad_z), _ptr(g), _ptr(rho), T, d,
                                         OUT_DTYPES[grad_x.dtype], _ptr(grad_x),
                                         _ptr(grad_gamma) if grad_gamma is not None else None,
                                         _stream(x.device)))
    return grad_x, grad_gamma


def mxnorm_linear_bwd(grad_h, x, rho, gamma, w, block=32, elem="e4m3",
                      grad_x_dtype=torch.bfloat16):
    """The MXNormLinear backward (Sec. 3.7; the implementation appendix's
    mx_norm_linear_backward), every product and cast in the library:
      grad_Z = MXCast(grad_H) MXCast_N(W)            (W blocked along N)
      grad_X, grad_gamma = STE(X, grad_Z, gamma, rho~)
      grad_W = (MXCast(grad_H^T) MXCast(rho~ X)^T) . gamma
    grad_h bf16 [T, N], x bf16 [T, d], rho float32 [T], gamma bf16 [d],
    w bf16 [N, d].  Returns (grad_x, grad_gamma float32 [d], grad_w float32
    [N, d])."""
    T, N = _input(grad_h)
    if _input(x)[0] != T:
        raise ValueError("x must have grad_h's rows")
    d = x.shape[1]
    if w.shape != (N, d):
        raise ValueError("w must be [N, d]")
    _input(w)
    if block not in (16, 32, 64) or elem not in ELEMS:
        raise ValueError("block must be 16, 32 or 64 and elem 'e4m3' or 'e2m1'")
    if x.device != grad_h.device or w.device != grad_h.device:
        raise ValueError("grad_h, x and w must be on one device")
    if rho.dtype != torch.float32 or rho.shape != (T,) or rho.device != x.device \
            or not rho.is_contiguous():
        raise ValueError("rho must be a contiguous float32 [T] tensor on x's device")
    if gamma is not None:
        _gamma(gamma, x)
        if not gamma.is_contiguous():
            raise ValueError("gamma must be contiguous")
    if grad_x_dtype not in OUT_DTYPES:
        raise ValueError("out_dtype must be float32 or bfloat16")
    lib, e = load(), ELEMS[elem]
    grad_x = torch.empty((T, d), dtype=grad_x_dtype, device=x.device)
    grad_gamma = torch.empty((d,), dtype=torch.float32, device=x.device)
    grad_w = torch.empty((N, d), dtype=torch.float32, device=x.device)
    ws_bytes = lib.mxnorm_linear_bwd_workspace_bytes(T, N, d, e)
    ws = torch.empty((ws_bytes,), dtype=torch.uint8, device=x.device)
    _check(lib.mxnorm_linear_bwd(grad_h.data_ptr(), x.data_ptr(), rho.data_ptr(), _ptr(gamma),
                                 w.data_ptr(), T, N, d, block, e, OUT_DTYPES[grad_x_dtype],
                                 grad_x.data_ptr(), grad_gamma.data_ptr(), grad_w.data_ptr(),
                                 ws.data_ptr(), ws_bytes, _stream(x.device)))
    return grad_x, grad_gamma, grad_w


class _Heads(ctypes.Structure):
    """mx_heads of include/mxnorm.h."""
    _fields_ = [("data", ctypes.c_void_p), ("heads", ctypes.c_int64),
                ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


def _heads(t, name, like=None):
    """A tensor of heads [T, H, D] by its strides; shaped as `like` if given."""
    if not isinstance(t, torch.Tensor) or t.dtype != torch.bfloat16 or t.dim() != 3:
        raise TypeError("%s must be a 3-D torch.bfloat16 tensor [T, heads, D]" % name)
    if not t.is_cuda:
        raise RuntimeError("%s must be on the GPU: libmxnorm has no CPU path" % name)
    if like is not None and (t.shape != like.shape or t.device != like.device):
        raise ValueError("%s must have the shape and device of its input" % name)
    st, sh, se = t.stride()
    if se != 1 and t.shape[2] > 1:
        raise ValueError("%s: the elements of a head must be contiguous" % name)
    return _Heads(t.data_ptr(), t.shape[1], st, sh)


def _new_heads(t):
    """A contiguous tensor like t and its mx_heads (empty_like: 1 us a tensor
    less than empty with a shape, type and device)."""
    out = torch.empty_like(t, memory_format=torch.contiguous_format)
    _, H, D = t.shape
    return out, _Heads(out.data_ptr(), H, H * D, D)


def _rope_arguments(q, k, q_gamma, k_gamma, pos, inv_freq, rotary):
    """(T, D, R) of a call on queries q and keys k, its vectors checked."""
    T, _, D = q.shape
    Tk, _, Dk = k.shape
    device = q.device
    if Tk != T or Dk != D or k.device != device:
        raise ValueError("q and k must have the same tokens, head size and device")
    for g, name in ((q_gamma, "q_gamma"), (k_gamma, "k_gamma")):
        if g is not None and (g.dtype != torch.bfloat16 or g.shape != (D,) or g.device != device
                              or not g.is_contiguous()):
            raise ValueError("%s must be a contiguous bfloat16 [D] tensor on q's device" % name)
    R = D if rotary is None else rotary
    if pos is not None and (pos.dtype != torch.int64 or pos.shape != (T,) or pos.device != device
                            or not pos.is_contiguous()):
        raise ValueError("pos must be a contiguous int64 [T] tensor on q's device")
    if R and (inv_freq is None or inv_freq.dtype != torch.float32 or inv_freq.shape != (R // 2,)
              or inv_freq.device != device or not inv_freq.is_contiguous()):
        raise ValueError("inv_freq must be a contiguous float32 [rotary / 2] tensor on q's device")
    return T, D, R


def qk_norm_rope_fwd(q, k, q_gamma, k_gamma, pos, inv_freq, rotary=None, interleaved=False, eps=1e-6,
                     q_out=None, k_out=None):
    """RMSNorm of every head of q [T, Hq, D] and k [T, Hk, D] with its gain (bf16
    [D] or None) and the rotation of its first `rotary` (None: all) elements by
    pos [T] (int64; None: 0, 1, ...) times inv_freq [rotary / 2] (float32), pairs
    (i, i + rotary / 2) or, interleaved, (2i, 2i + 1).  q and k may be views of
    a fused projection's output; q_out and k_out views of any buffer, q and k
    themselves among them.  Returns (q_out, k_out)."""
    dq, dk = _heads(q, "q"), _heads(k, "k")
    T, D, R = _rope_arguments(q, k, q_gamma, k_gamma, pos, inv_freq, rotary)
    q_out, oq = _new_heads(q) if q_out is None else (q_out, _heads(q_out, "q_out", q))
    k_out, ok = _new_heads(k) if k_out is None else (k_out, _heads(k_out, "k_out", k))
    ref = ctypes.byref
    _call(load().qk_norm_rope_fwd, q.device, ref(dq), ref(dk), _ptr(q_gamma), _ptr(k_gamma), T, D, R,
          _ptr(pos), _ptr(inv_freq), int(bool(interleaved)), eps, ref(oq), ref(ok))
    return q_out, k_out


def qk_norm_rope_bwd(grad_q_out, grad_k_out, q, k, q_gamma, k_gamma, pos, inv_freq, rotary=None,
                     interleaved=False, eps=1e-6, grad_q=None, grad_k=None, want_grad_gamma=True):
    """The gradients of qk_norm_rope_fwd, q and k as it took them: (grad_q,
    grad_k, grad_q_gamma, grad_k_gamma).  grad_q and grad_k may be views of the
    fused projection's gradient, or the incoming gradients themselves; the gain
    gradients are float32 [D], None without a gain or with want_grad_gamma =
    False."""
    dq, dk = _heads(q, "q"), _heads(k, "k")
    T, D, R = _rope_arguments(q, k, q_gamma, k_gamma, pos, inv_freq, rotary)
    gq, gk = _heads(grad_q_out, "grad_q_out", q), _heads(grad_k_out, "grad_k_out", k)
    grad_q, oq = _new_heads(q) if grad_q is None else (grad_q, _heads(grad_q, "grad_q", q))
    grad_k, ok = _new_heads(k) if grad_k is None else (grad_k, _heads(grad_k, "grad_k", k))
    lib = load()
    gg = [q.new_empty((D,), dtype=torch.float32) if want_grad_gamma and g is not None else None
          for g in (q_gamma, k_gamma)]
    ws_bytes = lib.qk_norm_rope_bwd_workspace_bytes(T, D) if gg[0] is not None or gg[1] is not None else 0
    ws = q.new_empty((ws_bytes,), dtype=torch.uint8) if ws_bytes else None
    ref = ctypes.byref
    _call(lib.qk_norm_rope_bwd, q.device, ref(gq), ref(gk), ref(dq), ref(dk), _ptr(q_gamma),
          _ptr(k_gamma), T, D, R, _ptr(pos), _ptr(inv_freq), int(bool(interleaved)), eps, ref(oq),
          ref(ok), _ptr(gg[0]), _ptr(gg[1]), _ptr(ws), ws_bytes)
    return grad_q, grad_k, gg[0], gg[1]


def _starts(t, name, device, n=None):
    """An int32 vector of n elements, if given; None stays None."""
    if t is not None and (t.dtype is not torch.int32 or t.dim() != 1 or t.device != device or not t.is_contiguous()
                          or (n is not None and len(t) != n)):
        raise ValueError("%s must be a contiguous int32 tensor%s on q's device" % (name, "" if n is None else " [%d]" % n))
    return t


def _attn_arguments(q, k, v, q_start, k_start, scale):
    """(mx_heads of q, k, v; Tq, Tk, D, sequences, scale) of a call."""
    dq, dk, dv = _heads(q, "q"), _heads(k, "k"), _heads(v, "v", k)
    Tq, Hq, D = q.shape
    Tk, Hk, Dk = k.shape
    device = q.device
    if Dk != D or k.device != device or Hk == 0 or Hq % Hk:
        raise ValueError("k and v must have q's head size and device, and q a multiple of their heads")
    sequences = 1
    if q_start is not None:
        _starts(q_start, "q_start", device)
        sequences = q_start.shape[0] - 1
        _starts(k_start, "k_start", device, sequences + 1)
    elif k_start is not None:
        raise ValueError("k_start needs a q_start")
    return dq, dk, dv, Tq, Tk, D, sequences, D ** -0.5 if scale is None else scale


def window_attn_fwd(q, k, v, window=0, sinks=0, scale=None, q_start=None, k_start=None, out=None, lse=None,
                    want_lse=True):
    """Causal attention of q [T, Hq, D] over k and v [S, Hk, D] (views of a
    projection's output among them), packed sequences by q_start and k_start
    (int32 [sequences + 1]; k_start None: q_start, both None: one sequence whose
    queries are its last tokens).  Of the keys up to its own place a query sees
    the last `window` (0: all) and the first `sinks`.  scale None: D ** -0.5.
    Returns (out [T, Hq, D], lse float32 [Hq, T] or None)."""
    dq, dk, dv, T, S, D, B, scale = _attn_arguments(q, k, v, q_start, k_start, scale)
    out, do = _new_heads(q) if out is None else (out, _heads(out, "out", q))
    if want_lse:
        lse = _out(lse, (q.shape[1], T), torch.float32, q.device)
    ref = ctypes.byref
    _call(load().window_attn_fwd, q.device, ref(dq), ref(dk), ref(dv), T, S, D, _ptr(q_start), _ptr(k_start), B,
          window, sinks, scale, ref(do), _ptr(lse) if want_lse else None)
    return out, (lse if want_lse else None)


def window_attn_bwd(grad_out, q, k, v, out, lse, window=0, sinks=0, scale=None, q_start=None, k_start=None,
                    grad_q=None, grad_k=None, grad_v=None):
    """The gradients of window_attn_fwd from that of its output: q, k, v and the
    rest as it took them, out and lse as it gave them.  grad_q, grad_k and grad_v
    may be views of the projection's gradient.  Returns (grad_q, grad_k, grad_v)."""
    dq, dk, dv, T, S, D, B, scale = _attn_arguments(q, k, v, q_start, k_start, scale)
    dg, do = _heads(grad_out, "grad_out", q), _heads(out, "out", q)
    Hq, device = q.shape[1], q.device
    if lse.shape != (Hq, T) or lse.dtype != torch.float32 or lse.device != device or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 [Hq, T] tensor on q's device")
    grad_q, gq = _new_heads(q) if grad_q is None else (grad_q, _heads(grad_q, "grad_q", q))
    grad_k, gk = _new_heads(k) if grad_k is None else (grad_k, _heads(grad_k, "grad_k", k))
    grad_v, gv = _new_heads(v) if grad_v is None else (grad_v, _heads(grad_v, "grad_v", v))
    lib = load()
    ws_bytes = lib.window_attn_bwd_workspace_bytes(T, S, Hq, k.shape[1], D, B, window, sinks)
    ws = q.new_empty((ws_bytes,), dtype=torch.uint8) if ws_bytes else None
    ref = ctypes.byref
    _call(lib.window_attn_bwd, device, ref(dg), ref(dq), ref(dk), ref(dv), ref(do), _ptr(lse), T, S, D,
          _ptr(q_start), _ptr(k_start), B, window, sinks, scale, ref(gq), ref(gk), ref(gv), _ptr(ws), ws_bytes)
    return grad_q, grad_k, grad_v


class _Cache(ctypes.Structure):
    """mx_kv_cache of include/mxnorm.h."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "k_scales", "v_scales")]
                + [(n, ctypes.c_int64) for n in ("pages", "page_size", "heads", "page_stride", "scale_page_stride")]
                + [("type", ctypes.c_int)])


def _paged(t, name, dtype, shape, device, page):
    """The page stride of pages whose slots are contiguous (0 of one page alone, which
    has no use for it); page: their strides."""
    strides = t.stride()
    if t.dtype != dtype or t.shape != shape or t.device != device or (strides[1:] != page and not t[:1].is_contiguous()):
        raise ValueError("%s must be %s %s on q's device, every page contiguous" % (name, dtype, list(shape)))
    return strides[0] if shape[0] > 1 else 0


def _cache(k_cache, v_cache, k_scales, v_scales, table, length, start, T, D, device):
    """(mx_kv_cache, table width, sequences) of a call."""
    dtype = k_cache.dtype
    mx = dtype is torch.uint8
    if k_cache.dim() != 4 or not (mx or dtype is torch.bfloat16):
        raise TypeError("k_cache must be [pages, heads, slots, D], torch.bfloat16, or torch.uint8 for E4M3 codes")
    if not k_cache.is_cuda:
        raise RuntimeError("k_cache must be on the GPU: libmxnorm has no CPU path")
    shape = k_cache.shape
    pages, heads, slots, Dc = shape
    page = (slots * Dc, Dc, 1)
    stride = _paged(k_cache, "k_cache", dtype, shape, device, page)
    if Dc != D or _paged(v_cache, "v_cache", dtype, shape, device, page) != stride:
        raise ValueError("k_cache and v_cache must have the head size of the call and the same pages")
    if mx != (k_scales is not None) or mx != (v_scales is not None):
        raise ValueError("k_scales and v_scales belong to E4M3 codes")
    scale_stride = 0
    if mx:
        n = D // 32
        scales, page = (pages, heads, slots, n), (slots * n, n, 1)
        scale_stride = _paged(k_scales, "k_scales", dtype, scales, device, page)
        if _paged(v_scales, "v_scales", dtype, scales, device, page) != scale_stride:
            raise ValueError("k_scales and v_scales must have the same pages")
    if table.dim() != 2 or table.dtype is not torch.int32 or table.device != device or not table.is_contiguous():
        raise ValueError("table must be a contiguous int32 [sequences, pages] tensor on q's device")
    B, width = table.shape
    _starts(length, "length", device, B)
    _starts(start, "start", device, B + 1)
    if start is None and T != B:
        raise ValueError("without start every sequence has one new token")
    return _Cache(k_cache.data_ptr(), v_cache.data_ptr(), _ptr(k_scales), _ptr(v_scales), pages, slots, heads, stride,
                  scale_stride, int(mx)), width, B


def kv_cache_append(k, v, k_cache, v_cache, table, length, start=None, rows=None, k_scales=None, v_scales=None):
    """New tokens' keys and values k, v [S, heads, D] into a paged cache, in place.

    k_cache, v_cache [pages, heads, slots, D]: bf16, or uint8 E4M3 codes with
    k_scales, v_scales uint8 [pages, heads, slots, D / 32] (E8M0).  Sequence b's
    new tokens start[b] .. start[b + 1] - 1 (int32 [sequences + 1]; None: one a
    sequence) go to places length[b] + i, in pages table[b] (int32 [sequences, n];
    a page that the cache does not have is skipped).  rows int32 or None: the row
    of k and v of every new token.  Returns (k_cache, v_cache), with scales
    (k_cache, k_scales, v_cache, v_scales)."""
    dk, dv = _heads(k, "k"), _heads(v, "v", k)
    S, heads, D = k.shape
    device = k.device
    _starts(rows, "rows", device)
    T = S if rows is None else rows.shape[0]
    if start is None and rows is None:
        T = table.shape[0]
    cache, width, B = _cache(k_cache, v_cache, k_scales, v_scales, table, length, start, T, D, device)
    ref = ctypes.byref
    _call(load().kv_cache_append, device, ref(cache), ref(dk), ref(dv), T, S, D, _ptr(table), width, _ptr(length),
          _ptr(start), B, _ptr(rows))
    return (k_cache, v_cache) if k_scales is None else (k_cache, k_scales, v_cache, v_scales)


def kv_cache_attn_fwd(q, k_cache, v_cache, table, length, start=None, max_new=None, ancestors=None, window=0, sinks=0,
                      scale=None, max_length=0, k_scales=None, v_scales=None, out=None):
    """Attention of new tokens q [T, Hq, D] over the cache that kv_cache_append
    has written them to (its arguments; length does not count them).

    start None: one new token a sequence; else max_new bounds their number (None:
    64, the most).  ancestors int64 [T] or None: bit u of a token's says that it
    sees drafted token u of its sequence (its own bit included); None: those up to
    itself.  window, sinks and scale as in window_attn_fwd, places counted along a
    token's own branch.  max_length: a bound of length, if the caller knows one (0:
    the table's room).  Returns out [T, Hq, D]."""
    dq = _heads(q, "q")
    T, Hq, D = q.shape
    device = q.device
    cache, width, B = _cache(k_cache, v_cache, k_scales, v_scales, table, length, start, T, D, device)
    if ancestors is not None and (ancestors.dtype != torch.int64 or ancestors.shape != (T,) or ancestors.device != device
                                  or not ancestors.is_contiguous()):
        raise ValueError("ancestors must be a contiguous int64 [T] tensor on q's device")
    if max_new is None:
        max_new = 1 if start is None else 64
    out, do = _new_heads(q) if out is None else (out, _heads(out, "out", q))
    lib = load()
    ws_bytes = lib.kv_cache_attn_fwd_workspace_bytes(T, Hq, cache.heads, D, B, cache.page_size, width, max_new, max_length,
                                                     window, sinks)
    ws = q.new_empty((ws_bytes,), dtype=torch.uint8) if ws_bytes else None
    ref = ctypes.byref
    _call(lib.kv_cache_attn_fwd, device, ref(cache), ref(dq), T, D, _ptr(table), width, _ptr(length), _ptr(start), B,
          max_new, max_length, _ptr(ancestors), window, sinks, D ** -0.5 if scale is None else scale, ref(do), _ptr(ws),
          ws_bytes)
    return out


def mxnorm_default_global_scale(d, block=16, p=2, coef=0.0):
    return float(load().mxnorm_default_global_scale(d, block, p, coef))


def rmsnorm_default_global_scale(d, gamma_absmax=1.0):
    return float(load().rmsnorm_default_global_scale(d, gamma_absmax))


def mxnorm_coef(block, p):
    return float(load().mxnorm_coef(block, p))


def mx_status_str(status):
    return load().mx_status_str(status).decode()


def mx_last_error():
    return load().mx_last_error().decode()
