"""Calls of one kernel of the library, past the choice that its entry points make
(mec_internal.h), and that choice itself."""
import ctypes

import torch

import paper_1706_06873_amd as mec

SMALL, FIRST, PATCH, TILE, FIXED = range(5)           # GemmKernel
WGRAD_TILE, WGRAD_SLAB, WGRAD_GENERAL = range(3)      # WgradKernel
UNSUPPORTED = -5
ALIGNED = 0x100000

_i, _vp = ctypes.c_int, ctypes.c_void_p
_lib = mec.lib
_lib.mec_internal_gemm_route.argtypes = [_vp, _vp] + [_i] * 11 + [ctypes.POINTER(_i)]
_lib.mec_internal_wgrad_route.argtypes = [_i] * 9
_lib.mec_internal_gemm.argtypes = [_i, _vp, _vp, _vp] + [_i] * 11 + [_vp]
_lib.mec_internal_wgrad.argtypes = [_i, _vp, _vp, _vp, _vp, ctypes.c_size_t] + [_i] * 10 + [_vp]
_lib.mec_internal_dgrad_gemm.argtypes = [_i, _vp, _vp, _vp] + [_i] * 9 + [_vp]


def route(dims, dtype="f32", algo="lowered", I=ALIGNED, K=ALIGNED):
    """(the kernel that the products of conv2d, or of gemm, take, whether they read I)."""
    from_input = _i(0)
    code = mec.F32 if dtype == "f32" else mec.BF16
    kind = {"lowered": mec.LOWERED, "fused": mec.FUSED, "gemm": -1}[algo]
    r = _lib.mec_internal_gemm_route(I, K, *dims, code, kind, ctypes.byref(from_input))
    assert r >= 0, (dims, r)
    return r, bool(from_input.value)


def wgrad_route(dims):
    r = _lib.mec_internal_wgrad_route(*dims)
    assert r >= 0, (dims, r)
    return r


def gemm(kernel, A, K, dims, fused, O=None):
    """O by one kernel from A (I if fused, else L), or None where it does not hold the
    shape."""
    i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w = dims
    o_h, o_w = mec.output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if O is None:
        O = torch.full((i_n, o_h, o_w, k_c), 7.0, device=A.device)
    r = _lib.mec_internal_gemm(kernel, A.data_ptr(), K.data_ptr(), O.data_ptr(), *dims,
                               mec.BF16 if A.dtype == torch.bfloat16 else mec.F32, int(fused),
                               torch.cuda.current_stream().cuda_stream)
    assert r in (0, UNSUPPORTED), (dims, r)
    return O if r == 0 else None


def wgrad(kernel, A, G, dims, fused):
    i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w = dims
    dK = torch.full((k_h, k_w, i_c, k_c), 7.0, device=A.device)
    ws = torch.empty(mec.grad_workspace_bytes(*dims, grad_pass=mec.GRAD_KERNEL), dtype=torch.uint8, device=A.device)
    r = _lib.mec_internal_wgrad(kernel, A.data_ptr(), G.data_ptr(), dK.data_ptr(), ws.data_ptr(), ws.numel(), *dims,
                                int(fused), torch.cuda.current_stream().cuda_stream)
    assert r in (0, UNSUPPORTED), (dims, r)
    return dK if r == 0 else None


def dgrad_gemm(tile, G, K, dims):
    i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w = dims
    o_w = mec.output_dims(i_h, i_w, k_h, k_w, s_h, s_w)[1]
    dL = torch.full((i_n, o_w, i_h, k_w, i_c), 7.0, device=G.device)
    r = _lib.mec_internal_dgrad_gemm(int(tile), G.data_ptr(), K.data_ptr(), dL.data_ptr(), *dims,
                                     torch.cuda.current_stream().cuda_stream)
    assert r in (0, UNSUPPORTED), (dims, r)
    return dL if r == 0 else None


_i64 = ctypes.c_int64
_lib.mec_internal_product.argtypes = [_i, _i, _vp, _vp, _vp, _vp] + [_i] * 4 + [_i64] * 3 + [_i, _vp]
_lib.mec_internal_product_plan.argtypes = [_i] * 7
XK, XKT, XTK = range(3)                               # Layout


def product_plan(layout, dtype, M, N, K, batch=1, may_split=False):
    """(kernel, shares of the reduction) that a product of the layer operators takes."""
    r = _lib.mec_internal_product_plan(layout, mec.F32 if dtype == "f32" else mec.BF16, M, N, K, batch, int(may_split))
    return r % 16, r // 16


def product(kernel, layout, A, B, splits=1):
    """A B by one kernel (0 the small one, from 1 the tiles); A is [m][k] ([k][m] for XTK), B
    [k][n] ([n][k] for XKT). None where there is no such kernel."""
    K, M = A.shape if layout == XTK else A.shape[::-1]
    N = B.shape[0] if layout == XKT else B.shape[1]
    Y = torch.full((M, N), 7.0, dtype=A.dtype, device=A.device)
    part = torch.empty(splits * M * N, device=A.device) if splits > 1 else None
    r = _lib.mec_internal_product(kernel, layout, A.data_ptr(), B.data_ptr(), Y.data_ptr(),
                                  part.data_ptr() if splits > 1 else None, splits, M, N, K, A.stride(0), B.stride(0), N,
                                  mec.BF16 if A.dtype == torch.bfloat16 else mec.F32,
                                  torch.cuda.current_stream().cuda_stream)
    assert r in (0, UNSUPPORTED), (kernel, layout, A.shape, B.shape, r)
    return Y if r == 0 else None


class _Operands(ctypes.Structure):  # mec_internal_operands
    _fields_ = ([(n, _vp) for n in ("A", "B", "Y", "Z", "R", "bias", "part")] +
                [(n, _i64) for n in ("lda", "ldb", "ldy", "ldz", "ldr", "a_batch", "b_batch", "second")] +
                [(n, _i) for n in ("splits", "batch", "act", "res_first", "symmetric")] +
                [(n, ctypes.c_float) for n in ("alpha", "beta", "diag")])


_lib.mec_internal_product_with.argtypes = [_i] * 6 + [ctypes.POINTER(_Operands), _vp]


def product_with(kernel, layout, A, B, splits=1, R=None, bias=None, act="none", res_first=False, Z=False, alpha=1.0,
                 beta=1.0, diag=0.0, symmetric=False, second=0, batch=1, Y=None):
    """product() with an epilogue, in parts (second: bytes to dZ's other part) or for a stack (A
    and B batch x .., dense): Y, or (Y, Z); None where there is no such kernel."""
    a, b = (A[0], B[0]) if batch > 1 else (A, B)
    K, M = a.shape if layout == XTK else a.shape[::-1]
    N = b.shape[0] if layout == XKT else b.shape[1]
    stack = (batch,) if batch > 1 else ()
    if Y is None:
        Y = torch.full(stack + (M, N), 7.0, dtype=A.dtype, device=A.device)
    z = torch.full((M, N), 7.0, dtype=A.dtype, device=A.device) if Z else None
    part = torch.empty(splits * batch * M * N, device=A.device) if splits > 1 else None
    ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    o = _Operands(ptr(A), ptr(B), ptr(Y), ptr(z), ptr(R), ptr(bias), ptr(part), a.stride(0), b.stride(0), Y.stride(-2), N,
                  R.stride(-2) if R is not None else 0, A.stride(0) if batch > 1 else 0, B.stride(0) if batch > 1 else 0,
                  second, splits, batch, mec._ACTS[act], int(res_first), int(symmetric), alpha, beta, diag)
    r = _lib.mec_internal_product_with(kernel, layout, mec.BF16 if A.dtype == torch.bfloat16 else mec.F32, M, N, K,
                                       ctypes.byref(o), torch.cuda.current_stream().cuda_stream)
    assert r in (0, UNSUPPORTED), (kernel, layout, A.shape, B.shape, r)
    return None if r else (Y, z) if Z else Y


_lib.mec_internal_orth_pairs.argtypes = [_i] * 4 + [ctypes.c_float] * 3


def orth_pairs(batch, rows, cols, steps=5, coefficients=(3.4445, -4.7750, 2.0315)):
    """Whether an orthogonalisation takes its first and its last two steps as one."""
    return bool(_lib.mec_internal_orth_pairs(batch, rows, cols, steps, *coefficients))


def orth_plan(batch, rows, cols, gram=True):
    """(kernel, shares) of an orthogonalisation's Gram matrices, or of its products of two squares."""
    r = _lib.mec_internal_orth_plan(batch, rows, cols, int(gram))
    return r % 16, r // 16


def linear_grad_route(rows, i_c, k_c, dtype, act="none"):
    """(how dX and dK are computed: 0 apart, 1 a pair of small ones, 2 a pair of tiles; dK's shares)."""
    r = _lib.mec_internal_linear_grad_route(rows, i_c, k_c, mec.F32 if dtype == "f32" else mec.BF16, mec._ACTS[act])
    return r % 16, r // 16
