"""MI355X (gfx950) multi-component floating-point (MCF) arithmetic.

Python binding of the C ABI in include/mcf.h (libmcf.so, built in-tree by
``paper_2207_08867_amd.build``).  This module only marshals arguments: it checks
shapes, dtypes and devices of torch tensors, passes their device pointers and the
current HIP stream, and turns status codes into exceptions.  Every arithmetic step
runs in the library's HIP kernels; there is no fallback.

Tensor conventions (component-major):
  * an MC tensor with nc components and logical shape S is a torch tensor of shape
    (nc, *S); a plain tensor has shape S or (1, *S);
  * component dtype torch.float16, torch.float32 or torch.float64; all tensors contiguous and on
    the same GPU.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os

__all__ = [
    "mc_add", "mc_mul", "mc_div", "mc_exp", "mc_renorm", "mc_matmul", "mc_matmul_splitk",
    "mc_matmul_splitk_slices", "mc_matmul_splitk_workspace", "mc_matmul_splitk_noalloc", "mc_linear_fwd", "mc_status_str",
    "mc_matmul_batched", "mc_bmm", "mc_addmm", "matmul_mcn", "mc_mul_slow", "mc_square", "mc_matmul_pruned",
    "mc_matmul_exact", "mc_matmul_exact_workspace", "mc_linreg_workspace", "mc_linreg_gd_step",
    "mc_linear_fwd_exact", "mc_linear_bwd", "mc_linear_bwd_workspace", "lib", "LIB_PATH", "MCFError",
    "mc_mx4_quantize", "mc_mx4_dequantize", "mc_mx4_matmul", "mc_mx4_matmul_workspace", "mc_mx4_linear_fwd",
    "mc_mx4_linear_fwd_workspace", "mc_mx4_linear_bwd", "mc_mx4_linear_bwd_workspace", "mc_distill_fwd",
    "mc_distill_bwd", "mc_distill_fwd_bwd", "mc_distill_workspace",
    "mc_rmsnorm_fwd", "mc_rmsnorm_int8", "mc_rmsnorm_bwd", "mc_rmsnorm_bwd_workspace", "mc_int8_quantize",
    "mc_int8_dequantize", "mc_int8_matmul", "mc_int8_matmul_workspace", "mc_int8_linear_fwd",
    "mc_int8_linear_fwd_workspace", "mc_logprobs_fwd", "mc_logprobs_bwd", "mc_logprobs_workspace",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libmcf.so")
_lib = None

MCF_F16, MCF_F32, MCF_F64, MCF_F16S, MCF_BF16 = 0, 1, 2, 3, 4


class MCFError(RuntimeError):
    pass


def lib() -> ctypes.CDLL:
    """Load libmcf.so; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MCFError(f"{LIB_PATH} is missing: build it with `python -m paper_2207_08867_amd.build` "
                           "(or __graft_entry__.build())")
        _torch()  # first: the library then shares torch's HIP runtime instead of loading another
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, ci = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
        for name in ("mc_add", "mc_mul", "mc_div"):
            f = getattr(L, name)
            f.restype = ci
            f.argtypes = [ci, ci, i64, vp, ci, vp, ci, vp, vp]
        L.mc_mul_slow.restype = ci
        L.mc_mul_slow.argtypes = [ci, ci, i64, vp, vp, vp, vp]
        L.mc_square.restype = ci
        L.mc_square.argtypes = [ci, ci, i64, vp, vp, vp]
        L.mc_exp.restype = ci
        L.mc_exp.argtypes = [ci, ci, i64, vp, vp, vp]
        L.mc_renorm.restype = ci
        L.mc_renorm.argtypes = [ci, ci, ci, i64, vp, vp, ci, vp]
        L.mc_matmul.restype = ci
        L.mc_matmul.argtypes = [ci, ci, i64, i64, i64, vp, ci, vp, ci, vp, vp]
        L.mc_matmul_splitk.restype = ci
        L.mc_matmul_splitk.argtypes = [ci, ci, i64, i64, i64, vp, ci, vp, ci, i64, vp, i64, vp, vp]
        L.mc_matmul_splitk_noalloc.restype = ci
        L.mc_matmul_splitk_noalloc.argtypes = [ci, ci, i64, i64, i64, vp, ci, vp, ci, i64, vp, vp]
        L.mc_matmul_splitk_slices.restype = i64
        L.mc_matmul_splitk_slices.argtypes = [i64, i64, i64]
        L.mc_matmul_splitk_workspace.restype = i64
        L.mc_matmul_splitk_workspace.argtypes = [ci, ci, i64, i64, i64, ci, ci, i64]
        L.mc_matmul_pruned.restype = ci
        L.mc_matmul_pruned.argtypes = [ci, ci, i64, i64, i64, vp, vp, vp, vp]
        L.mc_matmul_batched.restype = ci
        L.mc_matmul_batched.argtypes = [ci, ci, i64, i64, i64, i64, i64, vp, ci, i64, i64, i64, vp, ci, i64, i64,
                                        i64, vp, vp]
        L.mc_addmm.restype = ci
        L.mc_addmm.argtypes = [ci, ci, i64, i64, i64, vp, ci, vp, ci, vp, i64, ctypes.c_double, ctypes.c_double,
                               vp, vp]
        L.mc_matmul_exact.restype = ci
        L.mc_matmul_exact.argtypes = [ci, ci, i64, i64, i64, vp, ci, vp, ci, ci, vp, i64, vp, vp]
        L.mc_linear_fwd_exact.restype = ci
        L.mc_linear_fwd_exact.argtypes = [ci, ci, i64, i64, i64, vp, vp, vp, vp, i64, vp, vp]
        L.mc_matmul_exact_workspace.restype = i64
        L.mc_matmul_exact_workspace.argtypes = [ci, ci, i64, i64, i64]
        L.mc_linreg_workspace.restype = i64
        L.mc_linreg_workspace.argtypes = [ci, ci, i64, i64]
        L.mc_linreg_gd_step.restype = ci
        L.mc_linreg_gd_step.argtypes = [ci, ci, i64, i64, vp, vp, vp, ctypes.c_double, vp, i64, vp, vp]
        L.mc_linear_bwd.restype = ci
        L.mc_linear_bwd.argtypes = [ci, ci, i64, i64, i64, vp, vp, vp, ci, vp, vp, vp, vp, i64, vp]
        L.mc_linear_bwd_workspace.restype = i64
        L.mc_linear_bwd_workspace.argtypes = [ci, ci, i64, i64, i64]
        L.mc_linear_fwd.restype = ci
        L.mc_linear_fwd.argtypes = [ci, ci, i64, i64, i64, vp, vp, vp, vp, vp]
        cd = ctypes.c_double
        for name, args, res in (
            ("mc_mx4_quantize", [ci, ci, ci, i64, i64, vp, vp, vp, vp], ci),
            ("mc_mx4_dequantize", [ci, ci, i64, i64, vp, vp, vp, vp], ci),
            ("mc_mx4_matmul", [ci, i64, i64, i64, vp, vp, ci, vp, vp, ci, vp, i64, vp, vp], ci),
            ("mc_mx4_matmul_workspace", [ci, i64, i64, i64, ci, ci], i64),
            ("mc_mx4_linear_fwd", [ci, ci, i64, i64, i64, vp, vp, vp, vp, vp, i64, vp, vp], ci),
            ("mc_mx4_linear_fwd_workspace", [ci, ci, i64, i64, i64], i64),
            ("mc_mx4_linear_bwd", [ci, ci, i64, i64, i64, vp, vp, vp, vp, vp, vp, vp, vp, i64, vp], ci),
            ("mc_mx4_linear_bwd_workspace", [ci, ci, i64, i64, i64], i64),
            ("mc_distill_fwd", [ci, ci, i64, i64, i64, vp, vp, vp, cd, vp, i64, vp, vp, vp], ci),
            ("mc_distill_bwd", [ci, ci, i64, i64, i64, vp, vp, vp, cd, vp, vp, vp, vp], ci),
            ("mc_distill_fwd_bwd", [ci, ci, i64, i64, i64, vp, vp, vp, cd, vp, vp, i64, vp, vp, vp], ci),
            ("mc_distill_workspace", [i64, i64], i64),
            ("mc_rmsnorm_fwd", [ci, ci, i64, i64, vp, vp, vp, cd, vp, vp, vp], ci),
            ("mc_rmsnorm_int8", [ci, ci, i64, i64, vp, vp, vp, cd, vp, vp, vp, vp], ci),
            ("mc_rmsnorm_bwd", [ci, ci, i64, i64, vp, vp, vp, vp, cd, vp, vp, vp, i64, vp], ci),
            ("mc_rmsnorm_bwd_workspace", [ci, i64, i64], i64),
            ("mc_int8_quantize", [ci, ci, i64, i64, vp, vp, vp, vp], ci),
            ("mc_int8_dequantize", [ci, i64, i64, vp, vp, vp, vp], ci),
            ("mc_int8_matmul", [ci, i64, i64, i64, vp, vp, vp, vp, vp, vp, i64, vp, vp], ci),
            ("mc_int8_matmul_workspace", [ci, i64, i64, i64], i64),
            ("mc_int8_linear_fwd", [ci, i64, i64, i64, vp, vp, vp, vp, vp, i64, vp, vp], ci),
            ("mc_int8_linear_fwd_workspace", [ci, i64, i64, i64], i64),
            ("mc_logprobs_fwd", [ci, ci, i64, i64, i64, i64, vp, vp, cd, vp, i64, vp, vp, vp, vp, vp, vp], ci),
            ("mc_logprobs_bwd", [ci, ci, i64, i64, i64, vp, vp, cd, vp, vp, vp, vp, vp], ci),
            ("mc_logprobs_workspace", [i64, i64, i64], i64),
        ):
            f = getattr(L, name)
            f.argtypes, f.restype = args, res
        L.mc_status_str.restype = ctypes.c_char_p
        L.mc_status_str.argtypes = [ci]
        _lib = L
    return _lib


def mc_status_str(status: int) -> str:
    return (_lib or lib()).mc_status_str(int(status)).decode()


def _check(status: int, what: str):
    if status != 0:
        msg = f"{what}: {mc_status_str(status)}"
        if status in (-1, -2, -3, -4, -5, -7, -8):
            raise ValueError(msg)
        raise MCFError(msg)


# A small call is host-bound: its kernels take 2 to 4 us, so what the binding does per call
# is most of its time.  The helpers below keep that short: torch is looked up once, device
# pointers and the stream are plain integers (the library's argument types convert them),
# and the current stream's handle is read without building a Stream object (a 7850-element
# MC-SGD update, two calls: 21 -> 15 us).
_DTYPE_CODES = {}
_PLAIN_CODES = {}  # the formats of the calls on low-precision tensors and on rows of logits
_torch_module = None
_raw_stream = None
_plain_tensor = None


def _torch():
    global _torch_module, _raw_stream, _plain_tensor
    if _torch_module is None:
        import torch

        _DTYPE_CODES.update({torch.float16: MCF_F16, torch.float32: MCF_F32, torch.float64: MCF_F64})
        _PLAIN_CODES.update({torch.float16: MCF_F16, torch.bfloat16: MCF_BF16, torch.float32: MCF_F32})
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _plain_tensor = torch.Tensor
        _torch_module = torch
    return _torch_module


def _code(t, scaled: bool) -> int:
    """Format code of a tensor; scaled=True: binary16 with scaled low components
    (component c stands for 2^(-11 c) times its stored value), float16 tensors only."""
    if scaled:
        if t.dtype != _torch().float16:
            raise TypeError("scaled components need float16 tensors")
        return MCF_F16S
    return _dtype_code(t)


def _dtype_code(t) -> int:
    code = _DTYPE_CODES.get(t.dtype)
    if code is None:
        _torch()
        code = _DTYPE_CODES.get(t.dtype)
        if code is None:
            raise TypeError(f"component dtype must be float16, float32 or float64, got {t.dtype}")
    return code


def _dev(t, name) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _stream(t) -> int:
    """Handle of the current stream of t's device."""
    torch = _torch()
    if _raw_stream is not None:
        return _raw_stream(t.get_device())
    return torch.cuda.current_stream(t.device).cuda_stream


def _empty(x, shape):
    """A result of x's type and device: a plain tensor also for operands of a Tensor subclass."""
    if type(x) is _plain_tensor:
        return x.new_empty(shape)
    return _torch().empty(shape, dtype=x.dtype, device=x.device)


def _same(x, y) -> bool:
    return x.dtype == y.dtype and x.get_device() == y.get_device()


def _logical_shape(t, nc, is_mc, name):
    shape = t.shape
    if is_mc:
        if not shape or shape[0] != nc:
            raise ValueError(f"{name}: MC operand must have shape (nc={nc}, ...), got {tuple(shape)}")
        return shape[1:]
    return shape


def _binary(fn_name, x, y, nc, x_mc, y_mc, out, scaled=False):
    if not _same(x, y):
        raise ValueError("operands must share dtype and device")
    sx = _logical_shape(x, nc, x_mc, "x")
    sy = _logical_shape(y, nc, y_mc, "y")
    # a plain operand given as (1, *S) is accepted as S
    if not x_mc and len(sx) == len(sy) + 1 and sx[0] == 1:
        sx = sx[1:]
    if not y_mc and len(sy) == len(sx) + 1 and sy[0] == 1:
        sy = sy[1:]
    if sx != sy:
        raise ValueError(f"shape mismatch: {sx} vs {sy}")
    n = math.prod(sx)
    if out is None:
        out = _empty(x, (nc, *sx))
    elif out.shape != (nc, *sx) or out.dtype != x.dtype:
        raise ValueError("out has the wrong shape or dtype")
    st = getattr(_lib or lib(), fn_name)(_code(x, scaled), nc, n, _dev(x, "x"), int(bool(x_mc)), _dev(y, "y"),
                                         int(bool(y_mc)), _dev(out, "out"), _stream(x))
    _check(st, fn_name)
    return out


def mc_add(x, y, *, nc: int, x_mc: bool = True, y_mc: bool = True, out=None, scaled: bool = False):
    """Add-MCN for (MC, MC); Grow-ExpN for (MC, T) and (T, MC).  scaled=True: float16
    components with scaled low components (MC, MC only)."""
    return _binary("mc_add", x, y, nc, x_mc, y_mc, out, scaled)


def mc_mul(x, y, *, nc: int, x_mc: bool = True, y_mc: bool = True, out=None, scaled: bool = False):
    """Mult-MCN (fast) for (MC, MC); ScalingN for (MC, T) and (T, MC).  scaled=True:
    float16 components with scaled low components ((MC, T) and (T, MC) only)."""
    return _binary("mc_mul", x, y, nc, x_mc, y_mc, out, scaled)


def mc_div(x, y, *, nc: int, x_mc: bool = True, y_mc: bool = True, out=None):
    """Div-MCN for (MC, MC); DivN for (T, MC); zero-padded divisor for (MC, T)."""
    return _binary("mc_div", x, y, nc, x_mc, y_mc, out)


def mc_mul_slow(x, y, *, nc: int, out=None):
    """Mult-MCN-Slow of two MC operands of the same shape (nc, ...)."""
    torch = _torch()
    if x.dtype != y.dtype or x.device != y.device or x.shape != y.shape or x.shape[0] != nc:
        raise ValueError("x and y must be MC operands (nc, ...) of one shape, dtype and device")
    n = x.numel() // nc
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out has the wrong shape or dtype")
    st = (_lib or lib()).mc_mul_slow(_dtype_code(x), nc, n, _dev(x, "x"), _dev(y, "y"), _dev(out, "out"), _stream(x))
    _check(st, "mc_mul_slow")
    return out


def mc_square(x, *, nc: int, out=None):
    """Square-MCN of an MC operand (nc, ...)."""
    torch = _torch()
    _logical_shape(x, nc, True, "x")
    n = x.numel() // nc
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out has the wrong shape or dtype")
    _check((_lib or lib()).mc_square(_dtype_code(x), nc, n, _dev(x, "x"), _dev(out, "out"), _stream(x)), "mc_square")
    return out


def mc_exp(x, *, nc: int, out=None):
    """Exp-MCN (every component format; the component exponential is correctly rounded)."""
    torch = _torch()
    s = _logical_shape(x, nc, True, "x")
    n = x.numel() // nc
    if out is None:
        out = torch.empty_like(x)
    elif out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError("out has the wrong shape or dtype")
    del s
    _check((_lib or lib()).mc_exp(_dtype_code(x), nc, n, _dev(x, "x"), _dev(out, "out"), _stream(x)), "mc_exp")
    return out


def mc_renorm(x, *, nc_out: int | None = None, mode: int = 0, out=None):
    """mode 0: Renormalize; mode 1: Simple-Renorm.  x: (nc_in, ...)."""
    torch = _torch()
    nc_in = x.shape[0]
    nc_out = nc_in if nc_out is None else nc_out
    n = x.numel() // nc_in if nc_in else 0
    if out is None:
        out = torch.empty((nc_out,) + tuple(x.shape[1:]), dtype=x.dtype, device=x.device)
    elif out.shape != (nc_out,) + tuple(x.shape[1:]) or out.dtype != x.dtype:
        raise ValueError("out has the wrong shape or dtype")
    st = (_lib or lib()).mc_renorm(_dtype_code(x), nc_in, nc_out, n, _dev(x, "x"), _dev(out, "out"), int(mode),
                                   _stream(x))
    _check(st, "mc_renorm")
    return out


def _mm_operands(A, B, nc, a_mc, b_mc, out):
    if not _same(A, B):
        raise ValueError("operands must share dtype and device")
    A3 = A if A.dim() == 3 else A.reshape((1,) + tuple(A.shape))
    B3 = B if B.dim() == 3 else B.reshape((1,) + tuple(B.shape))
    planes_a, M, K = A3.shape
    planes_b, K2, N = B3.shape
    if planes_a != (nc if a_mc else 1) or planes_b != (nc if b_mc else 1):
        raise ValueError("operand plane count does not match nc / kind")
    if K != K2:
        raise ValueError(f"inner dimensions differ: {K} vs {K2}")
    if out is None:
        out = _empty(A, (nc, M, N))
    elif out.shape != (nc, M, N) or out.dtype != A.dtype:
        raise ValueError("out has the wrong shape or dtype")
    return A3, B3, M, N, K, out


def mc_matmul(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, out=None, scaled: bool = False):
    """C = A B in MM-MCN order.  A: (nc|1, M, K), B: (nc|1, K, N) -> (nc, M, N).
    scaled=True: float16 components with scaled low components."""
    A3, B3, M, N, K, out = _mm_operands(A, B, nc, a_mc, b_mc, out)
    st = (_lib or lib()).mc_matmul(_code(A, scaled), nc, M, N, K, _dev(A3, "A"), int(bool(a_mc)), _dev(B3, "B"),
                         int(bool(b_mc)), _dev(out, "out"), _stream(A))
    _check(st, "mc_matmul")
    return out


def mc_matmul_pruned(A, B, *, nc: int, out=None):
    """Pruned MC x MC product: component b of B multiplies the first nc - b components
    of A (the products A^(a) B^(b) with a + b >= nc, of order u^nc, are left out),
    parts combined by Add-MCN.  Same error bound as mc_matmul, about half the work at
    nc = 3; not mc_matmul's bits.  A: (nc, M, K), B: (nc, K, N) -> (nc, M, N)."""
    A3, B3, M, N, K, out = _mm_operands(A, B, nc, True, True, out)
    st = (_lib or lib()).mc_matmul_pruned(_dtype_code(A), nc, M, N, K, _dev(A3, "A"), _dev(B3, "B"), _dev(out, "out"),
                                _stream(A))
    _check(st, "mc_matmul_pruned")
    return out


def mc_matmul_splitk_slices(M: int, N: int, K: int) -> int:
    """Default slice count of the K-split product for this shape."""
    s = (_lib or lib()).mc_matmul_splitk_slices(M, N, K)
    _check(int(s) if s < 0 else 0, "mc_matmul_splitk_slices")
    return int(s)


def mc_matmul_splitk_workspace(dtype_code: int, nc: int, M: int, N: int, K: int, a_mc: bool, b_mc: bool,
                               slices: int) -> int:
    """Workspace bytes the K-split product needs."""
    w = (_lib or lib()).mc_matmul_splitk_workspace(dtype_code, nc, M, N, K, int(bool(a_mc)), int(bool(b_mc)), slices)
    _check(int(w) if w < 0 else 0, "mc_matmul_splitk_workspace")
    return int(w)


def mc_matmul_splitk(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, slices: int = 0, out=None,
                     workspace=None):
    """C = A B with the reduction dealt round-robin to `slices` slices (0: the default
    for the shape), each summed in MM-MCN order, the slice sums combined by a
    pairwise Add-MCN tree.  Shapes as for mc_matmul.  `workspace`: an optional
    device byte tensor; one is allocated here when needed and not given."""
    torch = _torch()
    A3, B3, M, N, K, out = _mm_operands(A, B, nc, a_mc, b_mc, out)
    code = _dtype_code(A)
    wb = mc_matmul_splitk_workspace(code, nc, M, N, K, a_mc, b_mc, slices)
    if wb > 0 and workspace is None:
        workspace = torch.empty(wb, dtype=torch.uint8, device=A.device)
    wp = _dev(workspace, "workspace") if workspace is not None else None
    wn = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = (_lib or lib()).mc_matmul_splitk(code, nc, M, N, K, _dev(A3, "A"), int(bool(a_mc)), _dev(B3, "B"),
                                          int(bool(b_mc)), int(slices), wp, wn, _dev(out, "out"), _stream(A))
    _check(st, "mc_matmul_splitk")
    return out


def mc_matmul_splitk_noalloc(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, slices: int = 0, out=None):
    """mc_matmul_splitk without a workspace: the library's static per-device scratch
    (8 MiB) holds the partial tree roots, so nothing is allocated when `out` is
    given.  Raises ValueError (MCF_E_SCRATCH) when the call needs more scratch."""
    A3, B3, M, N, K, out = _mm_operands(A, B, nc, a_mc, b_mc, out)
    st = (_lib or lib()).mc_matmul_splitk_noalloc(_dtype_code(A), nc, M, N, K, _dev(A3, "A"), int(bool(a_mc)),
                                                  _dev(B3, "B"),
                                                  int(bool(b_mc)), int(slices), _dev(out, "out"), _stream(A))
    _check(st, "mc_matmul_splitk_noalloc")
    return out


def mc_matmul_exact_workspace(nc: int, M: int, N: int, K: int) -> int:
    """Workspace bytes the exact binary16 product needs."""
    w = (_lib or lib()).mc_matmul_exact_workspace(MCF_F16, nc, M, N, K)
    _check(int(w) if w < 0 else 0, "mc_matmul_exact_workspace")
    return int(w)


def mc_matmul_exact(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, b_trans: bool = False, out=None,
                    workspace=None):
    """The exact product of binary16 MC matrices split into nc components by
    successive rounding (int8 matrix cores).  A: (nc|1, M, K); B: (nc|1, K, N), or
    (nc|1, N, K) with b_trans -> (nc, M, N).  `workspace`: an optional device byte
    tensor; one is allocated here when not given."""
    torch = _torch()
    if b_trans:
        Bv = B if B.dim() == 3 else B.reshape((1,) + tuple(B.shape))
        A3, _, M, N, K, out = _mm_operands(A, Bv.transpose(1, 2), nc, a_mc, b_mc, out)
        B3 = Bv
    else:
        A3, B3, M, N, K, out = _mm_operands(A, B, nc, a_mc, b_mc, out)
    wb = mc_matmul_exact_workspace(nc, M, N, K)
    if workspace is None:
        workspace = torch.empty(max(wb, 1), dtype=torch.uint8, device=A.device)
    wn = workspace.numel() * workspace.element_size()
    st = (_lib or lib()).mc_matmul_exact(_dtype_code(A), nc, M, N, K, _dev(A3, "A"), int(bool(a_mc)), _dev(B3, "B"),
                               int(bool(b_mc)), int(bool(b_trans)), _dev(workspace, "workspace"), wn,
                               _dev(out, "out"), _stream(A))
    _check(st, "mc_matmul_exact")
    return out


def mc_linreg_workspace(dtype_code: int, nc: int, n: int, d: int) -> int:
    """Workspace bytes of one linear-regression gradient-descent step."""
    w = (_lib or lib()).mc_linreg_workspace(dtype_code, nc, n, d)
    _check(int(w) if w < 0 else 0, "mc_linreg_workspace")
    return int(w)


def mc_linreg_gd_step(X, y_neg, W, lr: float, *, loss=None, workspace=None):
    """One gradient-descent step of MC-Linear regression with the mean-squared error
    (see include/mcf.h).  X: (n, d) plain; y_neg: (n,) the negated targets; W: (nc, d)
    MC, updated in place; loss: optional (nc,) MC output, the loss before the update.
    `workspace`: an optional device byte tensor; one is allocated here when not given."""
    torch = _torch()
    if X.dim() != 2 or W.dim() != 2 or y_neg.dim() != 1:
        raise ValueError("X must be (n, d), W (nc, d), y_neg (n,)")
    n, d = X.shape
    nc = W.shape[0]
    if W.shape[1] != d or y_neg.shape[0] != n or X.dtype != W.dtype or y_neg.dtype != W.dtype:
        raise ValueError("shape or dtype mismatch")
    if loss is not None and (tuple(loss.shape) != (nc,) or loss.dtype != W.dtype):
        raise ValueError("loss must be (nc,) of W's dtype")
    code = _dtype_code(W)
    if workspace is None:
        workspace = torch.empty(mc_linreg_workspace(code, nc, n, d), dtype=torch.uint8, device=W.device)
    st = (_lib or lib()).mc_linreg_gd_step(code, nc, n, d, _dev(X, "X"), _dev(y_neg, "y_neg"), _dev(W, "W"), float(lr),
                                 _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                 None if loss is None else _dev(loss, "loss"), _stream(W))
    _check(st, "mc_linreg_gd_step")
    return W


def mc_linear_fwd_exact(x, W, b=None, *, out=None, workspace=None):
    """Exact MC-Linear forward y = x W^T + b for binary16 components (int8 matrix
    cores): the exact value of every output split into nc components by successive
    rounding.  x: (batch, in) plain, W: (nc, out, in), b: (nc, out) or None ->
    y: (nc, batch, out)."""
    torch = _torch()
    nc, O, I = W.shape
    if x.dim() != 2 or x.shape[1] != I:
        raise ValueError("x must be (batch, in)")
    if x.dtype != W.dtype or (b is not None and (b.dtype != W.dtype or tuple(b.shape) != (nc, O))):
        raise ValueError("dtype or bias shape mismatch")
    T = x.shape[0]
    if out is None:
        out = _empty(W, (nc, T, O))
    elif tuple(out.shape) != (nc, T, O) or out.dtype != W.dtype:
        raise ValueError("out has the wrong shape or dtype")
    if workspace is None:
        workspace = torch.empty(max(mc_matmul_exact_workspace(nc, T, O, I), 1), dtype=torch.uint8, device=W.device)
    st = (_lib or lib()).mc_linear_fwd_exact(_dtype_code(W), nc, T, I, O, _dev(x, "x"), _dev(W, "W"),
                                   None if b is None else _dev(b, "b"), _dev(workspace, "workspace"),
                                   workspace.numel() * workspace.element_size(), _dev(out, "out"), _stream(W))
    _check(st, "mc_linear_fwd_exact")
    return out


def mc_linear_fwd(x, W, b=None, *, out=None, scaled: bool = False):
    """MC-Linear forward y = x W^T + b.  x: (batch, in) plain, W: (nc, out, in),
    b: (nc, out) or None -> y: (nc, batch, out).  scaled=True: float16 W, b and y with
    scaled low components (x is a plain float16 tensor)."""
    torch = _torch()
    nc, O, I = W.shape
    if x.dim() != 2 or x.shape[1] != I:
        raise ValueError("x must be (batch, in)")
    if x.dtype != W.dtype or (b is not None and (b.dtype != W.dtype or tuple(b.shape) != (nc, O))):
        raise ValueError("dtype or bias shape mismatch")
    T = x.shape[0]
    if out is None:
        out = _empty(W, (nc, T, O))
    elif out.shape != (nc, T, O) or out.dtype != W.dtype:
        raise ValueError("out has the wrong shape or dtype")
    bp = _dev(b, "b") if b is not None else None
    st = (_lib or lib()).mc_linear_fwd(_code(W, scaled), nc, T, I, O, _dev(x, "x"), _dev(W, "W"), bp, _dev(out, "out"),
                             _stream(W))
    _check(st, "mc_linear_fwd")
    return out


def mc_linear_bwd_workspace(dtype_code: int, nc: int, batch: int, in_: int, out: int) -> int:
    w = (_lib or lib()).mc_linear_bwd_workspace(dtype_code, nc, batch, in_, out)
    _check(int(w) if w < 0 else 0, "mc_linear_bwd_workspace")
    return int(w)


def mc_linear_bwd(x, W, dY, *, dy_mc: bool = True, dx: bool = True, dw: bool = True, db: bool = True,
                  workspace=None):
    """MC-Linear backward: dX = dY W, dW = dY^T x, db = column sums of dY (MM-MCN order).
    x: (batch, in) plain, W: (nc, out, in), dY: (nc, batch, out) or plain (batch, out).
    Returns (dX (nc, batch, in), dW (nc, out, in), db (nc, out)), None for the outputs
    not requested.  `workspace`: optional device byte tensor (allocated here if needed)."""
    torch = _torch()
    nc, O, I = W.shape
    if x.dim() != 2 or x.shape[1] != I:
        raise ValueError("x must be (batch, in)")
    T = x.shape[0]
    if tuple(dY.shape) != ((nc, T, O) if dy_mc else (T, O)):
        raise ValueError(f"dY must be {(nc, T, O) if dy_mc else (T, O)}, got {tuple(dY.shape)}")
    if x.dtype != W.dtype or dY.dtype != W.dtype:
        raise ValueError("dtype mismatch")
    code = _dtype_code(W)
    outs = [_empty(W, (nc, T, I)) if dx else None, _empty(W, (nc, O, I)) if dw else None,
            _empty(W, (nc, O)) if db else None]
    if (dw or db) and workspace is None:
        workspace = torch.empty(max(mc_linear_bwd_workspace(code, nc, T, I, O), 1), dtype=torch.uint8,
                                device=W.device)
    wp = _dev(workspace, "workspace") if workspace is not None else None
    wn = workspace.numel() * workspace.element_size() if workspace is not None else 0
    ptr = [(_dev(o, "out") if o is not None else None) for o in outs]
    st = (_lib or lib()).mc_linear_bwd(code, nc, T, I, O, _dev(x, "x"), _dev(W, "W"), _dev(dY, "dY"), int(bool(dy_mc)),
                             ptr[0], ptr[1], ptr[2], wp, wn, _stream(W))
    _check(st, "mc_linear_bwd")
    return tuple(outs)


def _batch_strides(t, name, batch, rows, cols):
    """(plane, s1, s2) of operand t = (planes, *b, rows, cols), len(b) <= 2, broadcast to
    the two batch dimensions `batch` (size-1 or missing dimensions get stride 0)."""
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    b = tuple(t.shape[1:-2])
    t5 = t.reshape((t.shape[0],) + (1,) * (2 - len(b)) + b + (rows, cols)).expand(
        (t.shape[0],) + tuple(batch) + (rows, cols))
    plane = t.stride(0) if t.shape[0] > 1 else t.numel()
    return plane, t5.stride(1) if batch[0] > 1 else 0, t5.stride(2) if batch[1] > 1 else 0


def mc_matmul_batched(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, out=None):
    """Batched / broadcast product (BMM-MCN, 4DMM-MCN): A (nc|1, *ba, M, K) times
    B (nc|1, *bb, K, N), up to two batch dimensions each, broadcast as torch.matmul
    broadcasts them -> (nc, *batch, M, N).  Each matrix product is taken as
    mc_matmul takes it."""
    torch = _torch()
    if A.dtype != B.dtype or A.device != B.device:
        raise ValueError("operands must share dtype and device")
    if A.dim() < 3 or B.dim() < 3 or A.dim() > 5 or B.dim() > 5:
        raise ValueError("operands must be (planes, [b1,] [b2,] rows, cols)")
    if A.shape[0] != (nc if a_mc else 1) or B.shape[0] != (nc if b_mc else 1):
        raise ValueError("operand plane count does not match nc / kind")
    M, K = A.shape[-2:]
    K2, N = B.shape[-2:]
    if K != K2:
        raise ValueError(f"inner dimensions differ: {K} vs {K2}")
    try:
        batch = tuple(torch.broadcast_shapes(tuple(A.shape[1:-2]), tuple(B.shape[1:-2])))
    except RuntimeError as e:
        raise ValueError(f"batch dimensions do not broadcast: {e}") from None
    b2 = (1,) * (2 - len(batch)) + batch
    if out is None:
        out = torch.empty((nc,) + batch + (M, N), dtype=A.dtype, device=A.device)
    elif tuple(out.shape) != (nc,) + batch + (M, N) or out.dtype != A.dtype:
        raise ValueError("out has the wrong shape or dtype")
    ap, as1, as2 = _batch_strides(A, "A", b2, M, K)
    bp, bs1, bs2 = _batch_strides(B, "B", b2, K, N)
    st = (_lib or lib()).mc_matmul_batched(_dtype_code(A), nc, b2[0], b2[1], M, N, K, _dev(A, "A"), int(bool(a_mc)),
                                           ap, as1,
                                           as2, _dev(B, "B"), int(bool(b_mc)), bp, bs1, bs2, _dev(out, "out"), _stream(A))
    _check(st, "mc_matmul_batched")
    return out


def mc_bmm(A, B, *, nc: int, a_mc: bool = True, b_mc: bool = True, out=None):
    """BMM-MCN: A (nc|1, b, M, K), B (nc|1, b, K, N) -> (nc, b, M, N)."""
    if A.dim() != 4 or B.dim() != 4:
        raise ValueError("BMM operands are (planes, batch, rows, cols)")
    return mc_matmul_batched(A, B, nc=nc, a_mc=a_mc, b_mc=b_mc, out=out)


def mc_addmm(A, B, Y, *, nc: int, alpha: float = 1.0, beta: float = 1.0, a_mc: bool = True, b_mc: bool = False,
             out=None):
    """AddMM-MCN: Add-MCN(ScalingN(A B, alpha), ScalingN(Y, beta)).  A (nc|1, M, K),
    B (nc|1, K, N), Y (nc, M, N) or (nc, N) (added to every row); alpha and beta must
    be values of the component format.  The paper's AddMM multiplies an MC matrix by a
    plain one (the defaults a_mc=True, b_mc=False)."""
    A3, B3, M, N, K, out = _mm_operands(A, B, nc, a_mc, b_mc, out)
    if Y.dtype != A.dtype or Y.device != A.device:
        raise ValueError("Y must share dtype and device with A")
    if tuple(Y.shape) == (nc, M, N):
        y_rows = M
    elif tuple(Y.shape) == (nc, N):
        y_rows = 1
    else:
        raise ValueError(f"Y must be (nc, M, N) or (nc, N), got {tuple(Y.shape)}")
    st = (_lib or lib()).mc_addmm(_dtype_code(A), nc, M, N, K, _dev(A3, "A"), int(bool(a_mc)), _dev(B3, "B"),
                        int(bool(b_mc)), _dev(Y, "Y"), y_rows, float(alpha), float(beta), _dev(out, "out"),
                        _stream(A))
    _check(st, "mc_addmm")
    return out


def matmul_mcn(x, y, *, nc: int, x_mc: bool = True, y_mc: bool = False):
    """Matmul-MCN: dispatch on the logical ranks of x and y (the planes dimension
    excluded) as torch.matmul does -- Dot-MCN (1, 1), MV-MCN (2, 1), vector-matrix
    (1, 2), MM-MCN (2, 2), batched (BMM-MCN / 4DMM-MCN) otherwise, with a 1-D operand
    taken as a column (resp. row) that is dropped from the result."""
    rx = x.dim() - 1
    ry = y.dim() - 1
    if rx < 1 or ry < 1:
        raise ValueError("operands need at least one logical dimension")
    xv = x.unsqueeze(-2) if rx == 1 else x  # (.., 1, K)
    yv = y.unsqueeze(-1) if ry == 1 else y  # (.., K, 1)
    if xv.dim() == 3 and yv.dim() == 3:
        out = mc_matmul(xv, yv, nc=nc, a_mc=x_mc, b_mc=y_mc)
    else:
        out = mc_matmul_batched(xv.contiguous(), yv.contiguous(), nc=nc, a_mc=x_mc, b_mc=y_mc)
    if rx == 1:
        out = out.squeeze(-2)
    if ry == 1:
        out = out.squeeze(-1)
    return out


# MXFP4 tensors are pairs (codes, scales) of uint8 tensors: for a tensor of shape (*S, n) in nc
# components, G = ceil(n / 128), codes (nc, *S, 64 G) and scales (nc, G, *S, 4).  The layout is
# in include/mcf.h.


def _plain_code(dtype) -> int:
    code = _PLAIN_CODES.get(dtype)
    if code is None:
        _torch()
        code = _PLAIN_CODES.get(dtype)
        if code is None:
            raise TypeError(f"dtype must be float16, bfloat16 or float32, got {dtype}")
    return code


def _mx4(pair, n, name):
    """(nc, S, codes pointer, scales pointer) of an MXFP4 tensor of row length n."""
    codes, scales = pair
    u8 = (_torch_module or _torch()).uint8
    if codes.dtype is not u8 or scales.dtype is not u8:
        raise TypeError(f"{name}: codes and scales must be uint8")
    if codes.get_device() != scales.get_device():
        raise ValueError(f"{name}: codes and scales must be on one device")
    groups = (n + 127) // 128
    cs, ss = codes.shape, scales.shape
    if n < 0 or len(cs) < 2 or cs[-1] != 64 * groups or ss != (cs[0], groups, *cs[1:-1], 4):
        raise ValueError(f"{name}: codes {tuple(cs)} and scales {tuple(ss)} are not an MXFP4 tensor of rows of {n}")
    return cs[0], cs[1:-1], _dev(codes, name), _dev(scales, name)


def _device(t, other, name):
    if t.get_device() != other.get_device():
        raise ValueError(f"{name} must be on the other operands' device")


def _out(out, like, shape, dtype):
    if out is None:
        return like.new_empty(shape, dtype=dtype) if type(like) is _plain_tensor else \
            _torch().empty(shape, dtype=dtype, device=like.device)
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype or out.get_device() != like.get_device():
        raise ValueError("out has the wrong shape, dtype or device")
    return out


def _space(workspace, needed, like):
    """(tensor to keep, pointer, bytes) of a workspace, allocated here when needed and not given."""
    if workspace is None:
        if needed <= 0:
            return None, None, 0
        workspace = _out(None, like, (needed,), _torch_module.uint8)
        return workspace, workspace.data_ptr(), needed
    _device(workspace, like, "workspace")
    return workspace, _dev(workspace, "workspace"), workspace.numel() * workspace.element_size()


@functools.lru_cache(maxsize=4096)
def _bytes(name, *sizes) -> int:
    """Workspace bytes of a call, a function of its sizes alone."""
    needed = int(getattr(_lib or lib(), name)(*sizes))
    _check(needed if needed < 0 else 0, name)
    return needed


def mc_mx4_quantize(x, *, nc: int = 1, x_mc: bool = False, out=None):
    """x (*S, n), or with x_mc an MC value (planes, *S, n) -> its MXFP4 tensor (codes, scales)
    of nc components: each block of 32 along a row scaled by a power of two and rounded to
    E2M1, each component the rounding of what the ones before it leave."""
    code = _plain_code(x.dtype)
    shape = x.shape
    nc_in = 1
    if len(shape) < (2 if x_mc else 1):
        raise ValueError("x must be (*S, n), or (planes, *S, n) with x_mc")
    if nc < 1:
        raise ValueError("nc must be positive")
    if x_mc:
        nc_in, shape = shape[0], shape[1:]
    n, lead = shape[-1], shape[:-1]
    groups = (n + 127) // 128
    codes, scales = out or (None, None)
    u8 = _torch_module.uint8
    codes = _out(codes, x, (nc, *lead, 64 * groups), u8)
    scales = _out(scales, x, (nc, groups, *lead, 4), u8)
    st = (_lib or lib()).mc_mx4_quantize(code, nc_in, nc, math.prod(lead), n, _dev(x, "x"), _dev(codes, "codes"),
                                         _dev(scales, "scales"), _stream(x))
    _check(st, "mc_mx4_quantize")
    return codes, scales


def mc_mx4_dequantize(codes, scales, n: int, *, dtype, out=None):
    """The numbers (*S, n) an MXFP4 tensor stands for, in `dtype`."""
    nc, shape, cp, sp = _mx4((codes, scales), n, "codes and scales")
    out = _out(out, codes, (*shape, n), dtype)
    st = (_lib or lib()).mc_mx4_dequantize(_plain_code(dtype), nc, math.prod(shape), n, cp, sp, _dev(out, "out"),
                                           _stream(codes))
    _check(st, "mc_mx4_dequantize")
    return out


def mc_mx4_matmul_workspace(dtype, M: int, N: int, K: int, a_nc: int, b_nc: int) -> int:
    """Workspace bytes of mc_mx4_matmul."""
    return _bytes("mc_mx4_matmul_workspace", _plain_code(dtype), M, N, K, a_nc, b_nc)


def mc_mx4_matmul(a, b, K: int, *, dtype, out=None, workspace=None):
    """a b^T of two MXFP4 tensors (codes, scales) with M and N rows of K -> (M, N) of `dtype`.
    `workspace`: an optional device byte tensor; one is allocated here when needed and not given."""
    a_nc, sa, ac, asc = _mx4(a, K, "a")
    b_nc, sb, bc, bsc = _mx4(b, K, "b")
    _device(b[0], a[0], "b")
    if len(sa) != 1 or len(sb) != 1:
        raise ValueError("a and b must be MXFP4 tensors of matrices")
    M, N = sa[0], sb[0]
    out = _out(out, a[0], (M, N), dtype)
    keep, wp, wn = _space(workspace, mc_mx4_matmul_workspace(dtype, M, N, K, a_nc, b_nc), a[0])
    st = (_lib or lib()).mc_mx4_matmul(_plain_code(dtype), M, N, K, ac, asc, a_nc, bc, bsc, b_nc, wp, wn,
                                       _dev(out, "out"), _stream(a[0]))
    _check(st, "mc_mx4_matmul")
    return out


def mc_mx4_linear_fwd_workspace(dtype, nc: int, batch: int, in_: int, out: int) -> int:
    """Workspace bytes of mc_mx4_linear_fwd."""
    return _bytes("mc_mx4_linear_fwd_workspace", _plain_code(dtype), nc, batch, in_, out)


def mc_mx4_linear_fwd(x, W, b=None, *, out=None, workspace=None):
    """y = x W^T + b.  x: (batch, in) plain, W: the MXFP4 tensor (codes, scales) of an (out, in)
    weight, b: (out,) of x's dtype or None -> (batch, out).  `workspace`: an optional device byte
    tensor; one is allocated here when needed and not given."""
    if x.dim() != 2:
        raise ValueError("x must be (batch, in)")
    T, I = x.shape
    nc, s, wc, wsc = _mx4(W, I, "W")
    _device(W[0], x, "W")
    if len(s) != 1:
        raise ValueError("W must be the MXFP4 tensor of a matrix")
    O = s[0]
    if b is not None:
        _device(b, x, "b")
        if b.dtype != x.dtype or tuple(b.shape) != (O,):
            raise ValueError("dtype or bias shape mismatch")
    code = _plain_code(x.dtype)
    out = _out(out, x, (T, O), x.dtype)
    keep, wp, wn = _space(workspace, _bytes("mc_mx4_linear_fwd_workspace", code, nc, T, I, O), x)
    st = (_lib or lib()).mc_mx4_linear_fwd(code, nc, T, I, O, _dev(x, "x"), wc, wsc, None if b is None else _dev(b, "b"), wp, wn,
                                _dev(out, "out"), _stream(x))
    _check(st, "mc_mx4_linear_fwd")
    return out


def mc_mx4_linear_bwd_workspace(dtype, nc: int, batch: int, in_: int, out: int) -> int:
    """Workspace bytes of mc_mx4_linear_bwd with every gradient."""
    return _bytes("mc_mx4_linear_bwd_workspace", _plain_code(dtype), nc, batch, in_, out)


def mc_mx4_linear_bwd(x, W, dY, *, dx: bool = True, dw: bool = True, db: bool = True, workspace=None):
    """The gradients of mc_mx4_linear_fwd: dX = dY W (batch, in), dW = dY^T x (out, in), the
    gradient of the numbers W stands for, and db = column sums of dY (out,); None for those not
    requested.  `workspace`: an optional device byte tensor; one is allocated here when not given."""
    if x.dim() != 2:
        raise ValueError("x must be (batch, in)")
    T, I = x.shape
    nc, s, wc, wsc = _mx4(W, I, "W")
    _device(W[0], x, "W")
    _device(dY, x, "dY")
    if len(s) != 1:
        raise ValueError("W must be the MXFP4 tensor of a matrix")
    O = s[0]
    if tuple(dY.shape) != (T, O) or dY.dtype != x.dtype:
        raise ValueError(f"dY must be {(T, O)} of x's dtype, got {tuple(dY.shape)} of {dY.dtype}")
    code = _plain_code(x.dtype)
    outs = [_empty(x, (T, I)) if dx else None, _empty(x, (O, I)) if dw else None, _empty(x, (O,)) if db else None]
    keep, wp, wn = _space(workspace, _bytes("mc_mx4_linear_bwd_workspace", code, nc, T, I, O), x)
    st = (_lib or lib()).mc_mx4_linear_bwd(code, nc, T, I, O, _dev(x, "x"), wc, wsc, _dev(dY, "dY"),
                                *(None if o is None else o.data_ptr() for o in outs), wp, wn, _stream(x))
    _check(st, "mc_mx4_linear_bwd")
    return tuple(outs)


def _distill_args(z, ids, t, g):
    """(code, nc, rows, vocab, k) of a distillation call's tensors."""
    torch = _torch_module or _torch()
    nc = 1
    shape = z.shape
    if len(shape) == 2:
        rows, vocab = shape
    elif len(shape) == 3:
        nc, rows, vocab = shape
    else:
        raise ValueError("z must be (rows, vocab), or (nc, rows, vocab) of an MC value")
    if ids.dtype is not torch.int32:
        raise TypeError(f"ids must be int32, got {ids.dtype}")
    shape = ids.shape
    if len(shape) != 2 or shape[0] != rows or t.shape != shape or t.dtype is not z.dtype:
        raise ValueError("ids and t must be (rows, k), t of z's dtype")
    _device(ids, z, "ids")
    _device(t, z, "t")
    if g is not None:
        if g.dtype is not torch.float32 or g.shape != (rows,):
            raise ValueError("g must be (rows,) float32")
        _device(g, z, "g")
    return _plain_code(z.dtype), nc, rows, vocab, shape[1]


def mc_distill_workspace(rows: int, vocab: int) -> int:
    """Workspace bytes of mc_distill_fwd and mc_distill_fwd_bwd."""
    return _bytes("mc_distill_workspace", rows, vocab)


def mc_distill_fwd(z, ids, t, *, temperature: float = 1.0, workspace=None):
    """Distillation from a teacher's top logits (see include/mcf.h): the loss of every row,
    T^2 KL(softmax of the k teacher logits t at ids || softmax of z), at temperature T.  z: (rows,
    vocab) plain or (nc, rows, vocab) MC; ids: (rows, k) int32, an id outside the vocabulary is an
    unused entry; t: (rows, k).  Returns (loss (rows,), stats (rows, 2)), both float32; stats are
    for mc_distill_bwd."""
    torch = _torch()
    code, nc, rows, vocab, k = _distill_args(z, ids, t, None)
    loss = _out(None, z, (rows,), torch.float32)
    stats = _out(None, z, (rows, 2), torch.float32)
    keep, wp, wn = _space(workspace, _bytes("mc_distill_workspace", rows, vocab), z)
    st = (_lib or lib()).mc_distill_fwd(code, nc, rows, vocab, k, _dev(z, "z"), _dev(ids, "ids"), _dev(t, "t"),
                             float(temperature), wp, wn, loss.data_ptr(), stats.data_ptr(), _stream(z))
    _check(st, "mc_distill_fwd")
    return loss, stats


def mc_distill_bwd(z, ids, t, stats, g=None, *, temperature: float = 1.0, out=None):
    """The gradient (rows, vocab) of sum_r g_r loss_r with respect to z (of the planes' sum for
    an MC z) from mc_distill_fwd's stats.  g: (rows,) float32, or None for ones."""
    code, nc, rows, vocab, k = _distill_args(z, ids, t, g)
    if stats.dtype != _torch().float32 or tuple(stats.shape) != (rows, 2):
        raise ValueError("stats must be (rows, 2) float32")
    _device(stats, z, "stats")
    out = _out(out, z, (rows, vocab), z.dtype)
    st = (_lib or lib()).mc_distill_bwd(code, nc, rows, vocab, k, _dev(z, "z"), _dev(ids, "ids"), _dev(t, "t"),
                                        float(temperature), _dev(stats, "stats"), None if g is None else _dev(g, "g"),
                                        _dev(out, "out"), _stream(z))
    _check(st, "mc_distill_bwd")
    return out


def mc_distill_fwd_bwd(z, ids, t, g=None, *, temperature: float = 1.0, out=None, workspace=None):
    """(loss, gradient) of mc_distill_fwd and mc_distill_bwd in one pass over z."""
    torch = _torch()
    code, nc, rows, vocab, k = _distill_args(z, ids, t, g)
    loss = _out(None, z, (rows,), torch.float32)
    out = _out(out, z, (rows, vocab), z.dtype)
    keep, wp, wn = _space(workspace, _bytes("mc_distill_workspace", rows, vocab), z)
    st = (_lib or lib()).mc_distill_fwd_bwd(code, nc, rows, vocab, k, _dev(z, "z"), _dev(ids, "ids"), _dev(t, "t"),
                                 float(temperature), None if g is None else _dev(g, "g"), wp, wn, loss.data_ptr(),
                                 _dev(out, "out"), _stream(z))
    _check(st, "mc_distill_fwd_bwd")
    return loss, out


# 8-bit tensors are pairs (codes, scales): for a tensor of shape (*S, n), P = n rounded up to a
# multiple of 128, codes (*S, P) int8 and scales (*S) float32.  The layout is in include/mcf.h.


def _int8(pair, n, name):
    """(S, codes pointer, scales pointer) of an 8-bit tensor of row length n."""
    codes, scales = pair
    torch = _torch_module or _torch()
    if codes.dtype is not torch.int8 or scales.dtype is not torch.float32:
        raise TypeError(f"{name}: codes must be int8 and scales float32")
    if codes.get_device() != scales.get_device():
        raise ValueError(f"{name}: codes and scales must be on one device")
    cs, lead = codes.shape, scales.shape
    if n < 0 or cs != lead + ((n + 127) // 128 * 128,):
        raise ValueError(f"{name}: codes {tuple(cs)} and scales {tuple(lead)} are not an 8-bit tensor of rows of {n}")
    return lead, _dev(codes, name), _dev(scales, name)


def _int8_out(out, like, lead, n):
    codes, scales = out or (None, None)
    return (_out(codes, like, lead + ((n + 127) // 128 * 128,), _torch_module.int8),
            _out(scales, like, lead, _torch_module.float32))


def _planes(x, x_mc, name):
    """(nc, S, n) of a plain tensor (*S, n) or, with x_mc, an MC value (nc, *S, n)."""
    shape = x.shape
    if len(shape) < (2 if x_mc else 1):
        raise ValueError(f"{name} must be (*S, n), or (planes, *S, n) of an MC value")
    return (shape[0], shape[1:-1], shape[-1]) if x_mc else (1, shape[:-1], shape[-1])


def mc_int8_quantize(x, *, x_mc: bool = False, out=None):
    """x (*S, n), or with x_mc an MC value (planes, *S, n) -> its 8-bit tensor (codes, scales): a row's
    largest magnitude becomes 127, the other elements the nearest integers, ties to even."""
    code = _plain_code(x.dtype)
    nc, lead, n = _planes(x, x_mc, "x")
    codes, scales = _int8_out(out, x, lead, n)
    st = (_lib or lib()).mc_int8_quantize(code, nc, math.prod(lead), n, _dev(x, "x"), _dev(codes, "codes"),
                                          _dev(scales, "scales"), _stream(x))
    _check(st, "mc_int8_quantize")
    return codes, scales


def mc_int8_dequantize(codes, scales, n: int, *, dtype, out=None):
    """The numbers (*S, n) an 8-bit tensor stands for, in `dtype`."""
    lead, cp, sp = _int8((codes, scales), n, "codes and scales")
    code = _plain_code(dtype)
    out = _out(out, codes, lead + (n,), dtype)
    st = (_lib or lib()).mc_int8_dequantize(code, math.prod(lead), n, cp, sp, _dev(out, "out"), _stream(codes))
    _check(st, "mc_int8_dequantize")
    return out


def _bias(b, n, dtype, like):
    if b is None:
        return None
    _device(b, like, "bias")
    if b.dtype != dtype or tuple(b.shape) != (n,):
        raise ValueError("dtype or bias shape mismatch")
    return _dev(b, "bias")


def mc_int8_matmul_workspace(dtype, M: int, N: int, K: int) -> int:
    """Workspace bytes of mc_int8_matmul."""
    return _bytes("mc_int8_matmul_workspace", _plain_code(dtype), M, N, K)


def mc_int8_matmul(a, b, K: int, bias=None, *, dtype, out=None, workspace=None):
    """a b^T (+ bias) of two 8-bit tensors (codes, scales) with M and N rows of K -> (M, N) of
    `dtype`; bias (N,) of `dtype` or None.  `workspace`: an optional device byte tensor; one is
    allocated here when needed and not given."""
    code = _plain_code(dtype)
    sa, ac, asc = _int8(a, K, "a")
    sb, bc, bsc = _int8(b, K, "b")
    _device(b[0], a[0], "b")
    if len(sa) != 1 or len(sb) != 1:
        raise ValueError("a and b must be 8-bit tensors of matrices")
    M, N = sa[0], sb[0]
    bp = _bias(bias, N, dtype, a[0])
    out = _out(out, a[0], (M, N), dtype)
    keep, wp, wn = _space(workspace, _bytes("mc_int8_matmul_workspace", code, M, N, K), a[0])
    st = (_lib or lib()).mc_int8_matmul(code, M, N, K, ac, asc, bc, bsc, bp, wp, wn, _dev(out, "out"), _stream(a[0]))
    _check(st, "mc_int8_matmul")
    return out


def mc_int8_linear_fwd_workspace(dtype, batch: int, in_: int, out: int) -> int:
    """Workspace bytes of mc_int8_linear_fwd."""
    return _bytes("mc_int8_linear_fwd_workspace", _plain_code(dtype), batch, in_, out)


def mc_int8_linear_fwd(x, W, b=None, *, out=None, workspace=None):
    """y = x W^T + b, each row of x quantised to 8 bits on the way.  x: (batch, in) plain, W: the 8-bit
    tensor (codes, scales) of an (out, in) weight, b: (out,) of x's dtype or None -> (batch, out).
    `workspace`: an optional device byte tensor; one is allocated here when needed and not given."""
    if x.dim() != 2:
        raise ValueError("x must be (batch, in)")
    T, I = x.shape
    code = _plain_code(x.dtype)
    s, wc, wsc = _int8(W, I, "W")
    _device(W[0], x, "W")
    if len(s) != 1:
        raise ValueError("W must be the 8-bit tensor of a matrix")
    O = s[0]
    bp = _bias(b, O, x.dtype, x)
    out = _out(out, x, (T, O), x.dtype)
    keep, wp, wn = _space(workspace, _bytes("mc_int8_linear_fwd_workspace", code, T, I, O), x)
    st = (_lib or lib()).mc_int8_linear_fwd(code, T, I, O, _dev(x, "x"), wc, wsc, bp, wp, wn, _dev(out, "out"),
                                            _stream(x))
    _check(st, "mc_int8_linear_fwd")
    return out


def _like(t, h, shape, name):
    """Pointer of t, a tensor of h's dtype and device and of this shape; None for none."""
    if t is None:
        return None
    if t.dtype is not h.dtype or t.shape != shape or t.get_device() != h.get_device():
        raise ValueError(f"{name} must be {tuple(shape)} of h's dtype and device, got {tuple(t.shape)} of {t.dtype} on "
                         f"{t.device}")
    return _dev(t, name)


def _norm_stream(h, x, h_out):
    """(the stream behind the addition, its pointer for the call)."""
    if x is None:
        if h_out is not None:
            raise ValueError("h_out is the stream behind the addition of x, which is not given")
        return h, None
    h_out = _out(h_out, h, h.shape, h.dtype)
    return h_out, _dev(h_out, "h_out")


def mc_rmsnorm_fwd(h, w=None, *, x=None, eps: float = 1e-6, h_mc: bool = False, h_out=None, out=None):
    """Root-mean-square norm of a residual stream h, (*S, n) or with h_mc an MC value (planes, *S, n), with
    x (*S, n), a layer's output, added to the stream first (see include/mcf.h); w: (n,) or None for ones.
    Returns (y (*S, n), the stream behind the addition: h itself without x).  h_out may be h (in place)."""
    code = _plain_code(h.dtype)
    nc, lead, n = _planes(h, h_mc, "h")
    row = lead + (n,)
    wp, xp = _like(w, h, (n,), "w"), _like(x, h, row, "x")
    stream, sp = _norm_stream(h, x, h_out)
    out = _out(out, h, row, h.dtype)
    st = (_lib or lib()).mc_rmsnorm_fwd(code, nc, math.prod(lead), n, _dev(h, "h"), xp, wp, float(eps), sp,
                                        _dev(out, "out"), _stream(h))
    _check(st, "mc_rmsnorm_fwd")
    return out, stream


def mc_rmsnorm_int8(h, w=None, *, x=None, eps: float = 1e-6, h_mc: bool = False, h_out=None, out=None):
    """mc_rmsnorm_fwd with the output as an 8-bit tensor: ((codes, scales), the stream behind the addition)."""
    code = _plain_code(h.dtype)
    nc, lead, n = _planes(h, h_mc, "h")
    wp, xp = _like(w, h, (n,), "w"), _like(x, h, lead + (n,), "x")
    stream, sp = _norm_stream(h, x, h_out)
    codes, scales = _int8_out(out, h, lead, n)
    st = (_lib or lib()).mc_rmsnorm_int8(code, nc, math.prod(lead), n, _dev(h, "h"), xp, wp, float(eps), sp,
                                         _dev(codes, "codes"), _dev(scales, "scales"), _stream(h))
    _check(st, "mc_rmsnorm_int8")
    return (codes, scales), stream


def mc_rmsnorm_bwd_workspace(dtype, rows: int, n: int) -> int:
    """Workspace bytes of mc_rmsnorm_bwd with dw."""
    return _bytes("mc_rmsnorm_bwd_workspace", _plain_code(dtype), rows, n)


def mc_rmsnorm_bwd(h, w, dy, *, dh=None, eps: float = 1e-6, h_mc: bool = False, dx: bool = True, dw: bool = True,
                   workspace=None):
    """The gradients of mc_rmsnorm_fwd: (that of the stream the norm was taken of, (*S, n), which is the
    gradient of h and of x alike, that of w (n,)); None for those not requested.  h: that stream (what
    mc_rmsnorm_fwd returned with x), dy: (*S, n), dh: the gradient that reaches the stream from elsewhere, (*S, n)
    or None.  `workspace`: an optional device byte tensor; one is allocated here when not given."""
    code = _plain_code(h.dtype)
    nc, lead, n = _planes(h, h_mc, "h")
    rows, row = math.prod(lead), lead + (n,)
    wp, yp, gp = _like(w, h, (n,), "w"), _like(dy, h, row, "dy"), _like(dh, h, row, "dh")
    gx, gw = _empty(h, row) if dx else None, _empty(h, (n,)) if dw else None
    keep, sp, sn = _space(workspace, _bytes("mc_rmsnorm_bwd_workspace", code, rows, n) if dw else 0, h)
    st = (_lib or lib()).mc_rmsnorm_bwd(code, nc, rows, n, _dev(h, "h"), wp, yp, gp, float(eps),
                                        gx.data_ptr() if dx else None, gw.data_ptr() if dw else None, sp, sn, _stream(h))
    _check(st, "mc_rmsnorm_bwd")
    return gx, gw


def _logprobs_args(z, ids):
    """(code, nc, rows, vocab, given) of the tensors of a call on log probabilities."""
    shape = z.shape
    if len(shape) not in (2, 3):
        raise ValueError("z must be (rows, vocab), or (nc, rows, vocab) of an MC value")
    nc, (rows, vocab) = (shape[0] if len(shape) == 3 else 1), shape[-2:]
    if ids.dtype is not (_torch_module or _torch()).int32:
        raise TypeError(f"ids must be int32, got {ids.dtype}")
    if len(ids.shape) != 2 or ids.shape[0] != rows:
        raise ValueError(f"ids must be (rows = {rows}, given), got {tuple(ids.shape)}")
    _device(ids, z, "ids")
    return _plain_code(z.dtype), nc, rows, vocab, ids.shape[1]


def mc_logprobs_workspace(rows: int, vocab: int, top: int) -> int:
    """Workspace bytes of mc_logprobs_fwd."""
    return _bytes("mc_logprobs_workspace", rows, vocab, top)


def mc_logprobs_fwd(z, ids, *, top: int = 0, temperature: float = 1.0, workspace=None):
    """Log probabilities under softmax(z / temperature) of given tokens, with the entropy and the `top` most
    likely tokens of every row (see include/mcf.h).  z: (rows, vocab) plain or (nc, rows, vocab) MC; ids:
    (rows, given) int32, an id outside the vocabulary is no token.  Returns (logp (rows, given), entropy (rows,),
    top_ids (rows, top) int32, top_logp (rows, top), stats (rows, 3)), float32 but for the ids; stats are for
    mc_logprobs_bwd.  `workspace`: an optional device byte tensor; one is allocated here when needed and not given."""
    torch = _torch()
    code, nc, rows, vocab, given = _logprobs_args(z, ids)
    keep, wp, wn = _space(workspace, _bytes("mc_logprobs_workspace", rows, vocab, top), z)
    f32 = torch.float32
    logp, entropy, stats = _out(None, z, (rows, given), f32), _out(None, z, (rows,), f32), _out(None, z, (rows, 3), f32)
    top_ids, top_logp = _out(None, z, (rows, top), torch.int32), _out(None, z, (rows, top), f32)
    st = (_lib or lib()).mc_logprobs_fwd(code, nc, rows, vocab, given, top, _dev(z, "z"), _dev(ids, "ids"),
                                         float(temperature), wp, wn, logp.data_ptr(), entropy.data_ptr(),
                                         top_ids.data_ptr(), top_logp.data_ptr(), stats.data_ptr(), _stream(z))
    _check(st, "mc_logprobs_fwd")
    return logp, entropy, top_ids, top_logp, stats


def mc_logprobs_bwd(z, ids, stats, g=None, g_entropy=None, *, temperature: float = 1.0, out=None):
    """The gradient (rows, vocab) of sum g logp + sum g_entropy entropy with respect to z (of the planes' sum
    for an MC z) from mc_logprobs_fwd's stats.  g: (rows, given) float32 or None for ones; g_entropy: (rows,)
    float32 or None for zeros."""
    f32 = _torch().float32
    code, nc, rows, vocab, given = _logprobs_args(z, ids)
    for name, t, shape in (("stats", stats, (rows, 3)), ("g", g, (rows, given)), ("g_entropy", g_entropy, (rows,))):
        if t is None and name != "stats":
            continue
        if t.dtype != f32 or tuple(t.shape) != shape:
            raise ValueError(f"{name} must be {shape} float32")
        _device(t, z, name)
    out = _out(out, z, (rows, vocab), z.dtype)
    st = (_lib or lib()).mc_logprobs_bwd(code, nc, rows, vocab, given, _dev(z, "z"), _dev(ids, "ids"),
                                         float(temperature), _dev(stats, "stats"), None if g is None else _dev(g, "g"),
                                         None if g_entropy is None else _dev(g_entropy, "g_entropy"),
                                         _dev(out, "out"), _stream(z))
    _check(st, "mc_logprobs_bwd")
    return out
