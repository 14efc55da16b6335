"""MI355X (gfx950) MEC convolution: thin Python binding of ``include/mec.h``.

MEC is the memory-efficient convolution of Cho & Brand (ICML 2017): a compact
lowering of the input I into L (i_n x o_w x i_h x k_w x i_c), then o_h small
matrix products over overlapping slabs of L. Every step runs in the HIP kernels
of ``libmec.so``; this module only marshals arguments. PyTorch supplies device
memory and streams: tensors passed here must be contiguous tensors on a HIP
device. There is no CPU fallback: if the library is missing, importing this
package raises.

Layouts (paper notation): I is i_n x i_h x i_w x i_c, K is k_h x k_w x i_c x
k_c, O is i_n x o_h x o_w x k_c (fp32). I and K are both fp32 or both bf16.
"""
import ctypes
import functools
import os

# torch first: importing it loads its HIP runtime, and libmec.so then binds to
# that same runtime. Loaded the other way round, the process would map a
# second HIP runtime (the system one) beside torch's, and device memory and
# streams from one are not valid in the other.
import torch  # noqa: E402,F401

__all__ = [
    "MecError", "F32", "BF16", "LOWERED", "FUSED", "IM2COL", "lib", "output_dims",
    "workspace_bytes", "im2col_bytes", "lower", "im2col", "gemm", "conv2d", "strerror",
    "GRAD_INPUT", "GRAD_KERNEL", "GRAD_KERNEL_FROM_L", "grad_workspace_bytes", "fold",
    "dgrad_gemm", "conv2d_dgrad", "wgrad_gemm", "conv2d_wgrad", "noalloc_scratch_bytes",
    "conv2d_wgrad_noalloc",
    "linear", "linear_workspace_bytes", "linear_grad", "linear_grad_workspace_bytes", "layer_norm", "layer_norm_grad",
    "layer_norm_grad_workspace_bytes", "orthogonalize", "orthogonalize_workspace_bytes",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmec.so")

F32, BF16 = 0, 1
LOWERED, FUSED, IM2COL = 0, 1, 2
GRAD_INPUT, GRAD_KERNEL, GRAD_KERNEL_FROM_L = 0, 1, 2
_UNSUPPORTED = -5  # MEC_ERR_UNSUPPORTED
_ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
_ALGOS = {"lowered": LOWERED, "fused": FUSED, "im2col": IM2COL,
          LOWERED: LOWERED, FUSED: FUSED, IM2COL: IM2COL}

if not os.path.exists(LIB_PATH):
    raise ImportError("%s is not built; run `python paper_1706_06873_amd/build.py`" % LIB_PATH)

_i = ctypes.c_int
_vp = ctypes.c_void_p
_DIMS = [_i] * 9


def _load(path):
    L = ctypes.CDLL(path)
    L.mec_output_dims.argtypes = [_i] * 6 + [ctypes.POINTER(_i), ctypes.POINTER(_i)]
    L.mec_output_dims.restype = _i
    L.mec_workspace_bytes.argtypes = _DIMS + [_i, _i]
    L.mec_workspace_bytes.restype = ctypes.c_int64
    L.mec_im2col_bytes.argtypes = _DIMS + [_i]
    L.mec_im2col_bytes.restype = ctypes.c_int64
    L.mec_lower.argtypes = [_vp, _vp] + _DIMS + [_i, _vp]
    L.mec_lower.restype = _i
    L.mec_im2col.argtypes = [_vp, _vp] + _DIMS + [_i, _vp]
    L.mec_im2col.restype = _i
    L.mec_gemm.argtypes = [_vp, _vp, _vp] + _DIMS + [_i, _vp]
    L.mec_gemm.restype = _i
    L.mec_conv2d.argtypes = [_vp, _vp, _vp, _vp, ctypes.c_size_t] + _DIMS + [_i, _i, _vp]
    L.mec_conv2d.restype = _i
    L.mec_grad_workspace_bytes.argtypes = _DIMS + [_i, _i]
    L.mec_grad_workspace_bytes.restype = ctypes.c_int64
    L.mec_fold.argtypes = [_vp, _vp] + _DIMS + [_vp]
    L.mec_fold.restype = _i
    L.mec_dgrad_gemm.argtypes = [_vp, _vp, _vp] + _DIMS + [_i, _vp]
    L.mec_dgrad_gemm.restype = _i
    for name in ("mec_conv2d_dgrad", "mec_wgrad_gemm", "mec_conv2d_wgrad"):
        getattr(L, name).argtypes = [_vp, _vp, _vp, _vp, ctypes.c_size_t] + _DIMS + [_i, _vp]
        getattr(L, name).restype = _i
    L.mec_noalloc_scratch_bytes.argtypes = []
    L.mec_noalloc_scratch_bytes.restype = ctypes.c_int64
    L.mec_conv2d_wgrad_noalloc.argtypes = [_vp, _vp, _vp] + _DIMS + [_i, _vp]
    L.mec_conv2d_wgrad_noalloc.restype = _i
    i64, sz, f = ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    L.mec_linear.argtypes = [_vp] * 6 + [i64, _i, _i, i64, i64, i64, _i, _i, _i, _vp, sz, _vp]
    L.mec_linear_workspace_bytes.argtypes = [i64, _i, _i, _i]
    L.mec_linear_grad_workspace_bytes.argtypes = [i64, _i, _i, _i]
    L.mec_linear_grad_act_workspace_bytes.argtypes = [i64, _i, _i, _i, _i]
    L.mec_linear_grad_act_workspace_bytes.restype = i64
    L.mec_linear_grad.argtypes = [_vp] * 9 + [sz, i64, _i, _i, i64, i64, _i, _i, _vp]
    L.mec_layer_norm.argtypes = [_vp] * 6 + [i64, _i, i64, i64, f, _i, _vp]
    L.mec_layer_norm_grad_workspace_bytes.argtypes = [i64, _i, _i]
    L.mec_layer_norm_grad.argtypes = [_vp] * 9 + [sz, i64, _i, i64, i64, _i, _vp]
    L.mec_orthogonalize_workspace_bytes.argtypes = [_i] * 4
    L.mec_orthogonalize.argtypes = [_vp] * 3 + [sz, _i, _i, _i, _i, f, f, f, f, _i, _vp]
    for name in ("linear", "linear_grad", "layer_norm", "layer_norm_grad", "orthogonalize"):
        getattr(L, "mec_" + name).restype = _i
        if name != "layer_norm":
            getattr(L, "mec_%s_workspace_bytes" % name).restype = i64
    L.mec_strerror.argtypes = [_i]
    L.mec_strerror.restype = ctypes.c_char_p
    L.mec_last_error.argtypes = []
    L.mec_last_error.restype = ctypes.c_char_p
    return L


def _hip_runtimes():
    """Distinct HIP runtime libraries mapped into this process."""
    try:
        with open("/proc/self/maps") as f:
            paths = {line.split()[-1] for line in f if "libamdhip64" in line}
    except OSError:
        return []
    return sorted(os.path.realpath(p) for p in paths)


lib = _load(LIB_PATH)
if len(_hip_runtimes()) > 1:
    raise ImportError("two HIP runtimes are loaded in this process (%s): libmec.so must bind to "
                      "the one torch uses" % ", ".join(_hip_runtimes()))


class MecError(RuntimeError):
    """A negative status from the library."""

    def __init__(self, status, what):
        self.status = status
        detail = lib.mec_last_error().decode() if status == -4 else ""
        super().__init__("%s: %s (status %d)%s" % (what, strerror(status), status,
                                                    " -- " + detail if detail else ""))


def strerror(status):
    return lib.mec_strerror(status).decode()


def _check(status, what):
    if status < 0:
        raise MecError(int(status), what)
    return status


def output_dims(i_h, i_w, k_h, k_w, s_h, s_w):
    """(o_h, o_w) by Eq. (1), floor reading."""
    o_h, o_w = _i(), _i()
    _check(lib.mec_output_dims(i_h, i_w, k_h, k_w, s_h, s_w, ctypes.byref(o_h), ctypes.byref(o_w)),
           "mec_output_dims")
    return o_h.value, o_w.value


def _dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError("I and K must be float32 or bfloat16, got %s" % t.dtype)


def workspace_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype=F32, algo=LOWERED):
    return _check(lib.mec_workspace_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype,
                                          _ALGOS[algo]), "mec_workspace_bytes")


def im2col_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype=F32):
    return _check(lib.mec_im2col_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype),
                  "mec_im2col_bytes")


def _stream_handle(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev_ptr(t, name):
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return ctypes.c_void_p(t.data_ptr())


def _same_device(t, ref, name):
    if t.device != ref.device:
        raise ValueError("%s is on %s, the inputs on %s" % (name, t.device, ref.device))


def _check_out(t, shape, dtype, ref, name):
    """A caller-supplied output must have exactly the shape, dtype and device
    the kernels write, so they never write past its end."""
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype:
        raise ValueError("%s must be %s of shape %s, got %s of shape %s"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    _same_device(t, ref, name)


def _dims(I, K, s_h, s_w):
    if I.dim() != 4 or K.dim() != 4:
        raise ValueError("I must be i_n x i_h x i_w x i_c and K k_h x k_w x i_c x k_c")
    i_n, i_h, i_w, i_c = I.shape
    k_h, k_w, k_ic, k_c = K.shape
    if k_ic != i_c:
        raise ValueError("K's third dimension (%d) must equal i_c (%d)" % (k_ic, i_c))
    if I.dtype != K.dtype:
        raise TypeError("I and K must have the same dtype")
    _same_device(K, I, "K")
    return (i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w)


def lower(I, k_h, k_w, k_c, s_h, s_w, L=None, stream=None):
    """MEC lowering of I into L (i_n x o_w x i_h x k_w x i_c); returns L. A
    given L must hold exactly mec_workspace_bytes(..., LOWERED) bytes of I's
    dtype (any shape)."""
    import torch
    if I.dim() != 4:
        raise ValueError("I must be i_n x i_h x i_w x i_c")
    i_n, i_h, i_w, i_c = I.shape
    dt = _dtype_code(I)
    _, o_w = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    need = workspace_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype=dt, algo=LOWERED)
    if L is None:
        L = torch.empty((i_n, o_w, i_h, k_w, i_c), dtype=I.dtype, device=I.device)
    _same_device(L, I, "L")
    if L.numel() * L.element_size() != need or L.dtype != I.dtype:
        raise ValueError("L must hold %d bytes of %s" % (need, I.dtype))
    _check(lib.mec_lower(_dev_ptr(I, "I"), _dev_ptr(L, "L"), i_n, i_h, i_w, i_c, k_h, k_w, k_c,
                         s_h, s_w, dt, _stream_handle(stream)), "mec_lower")
    return L


def im2col(I, k_h, k_w, k_c, s_h, s_w, M=None, stream=None):
    """im2col lowering of I, rows in (n, x, y) order: M is
    i_n x o_w x o_h x k_h x k_w x i_c. Returns M. A given M must hold exactly
    mec_im2col_bytes bytes of I's dtype (any shape)."""
    import torch
    if I.dim() != 4:
        raise ValueError("I must be i_n x i_h x i_w x i_c")
    i_n, i_h, i_w, i_c = I.shape
    dt = _dtype_code(I)
    o_h, o_w = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    need = im2col_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype=dt)
    if M is None:
        M = torch.empty((i_n, o_w, o_h, k_h, k_w, i_c), dtype=I.dtype, device=I.device)
    _same_device(M, I, "M")
    if M.numel() * M.element_size() != need or M.dtype != I.dtype:
        raise ValueError("M must hold %d bytes of %s" % (need, I.dtype))
    _check(lib.mec_im2col(_dev_ptr(I, "I"), _dev_ptr(M, "M"), i_n, i_h, i_w, i_c, k_h, k_w, k_c,
                          s_h, s_w, dt, _stream_handle(stream)), "mec_im2col")
    return M


def _out(I, K, s_h, s_w, O):
    import torch
    d = _dims(I, K, s_h, s_w)
    o_h, o_w = output_dims(d[1], d[2], d[4], d[5], s_h, s_w)
    shape = (d[0], o_h, o_w, d[6])
    if O is None:
        O = torch.empty(shape, dtype=torch.float32, device=I.device)
    _check_out(O, shape, torch.float32, I, "O")
    return d, O


def gemm(L, K, i_h, i_w, s_h, s_w, O=None, stream=None):
    """MEC's slab products on a lowered L (i_n x o_w x i_h x k_w x i_c); returns O.
    K is k_h x k_w x i_c x k_c of L's dtype; a given O must be float32 of shape
    i_n x o_h x o_w x k_c."""
    import torch
    if L.dim() != 5 or K.dim() != 4:
        raise ValueError("L must be i_n x o_w x i_h x k_w x i_c and K k_h x k_w x i_c x k_c")
    i_n, o_w, l_ih, k_w, i_c = L.shape
    k_h, kk_w, k_ic, k_c = K.shape
    if l_ih != i_h or kk_w != k_w or k_ic != i_c:
        raise ValueError("L (%s) and K (%s) do not agree on i_h, k_w and i_c"
                         % (tuple(L.shape), tuple(K.shape)))
    if K.dtype != L.dtype:
        raise TypeError("L and K must have the same dtype")
    _same_device(K, L, "K")
    dt = _dtype_code(L)
    o_h, o_w2 = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if o_w2 != o_w:
        raise ValueError("L's o_w does not match i_w, k_w, s_w")
    shape = (i_n, o_h, o_w, k_c)
    if O is None:
        O = torch.empty(shape, dtype=torch.float32, device=L.device)
    _check_out(O, shape, torch.float32, L, "O")
    _check(lib.mec_gemm(_dev_ptr(L, "L"), _dev_ptr(K, "K"), _dev_ptr(O, "O"), i_n, i_h, i_w, i_c,
                        k_h, k_w, k_c, s_h, s_w, dt, _stream_handle(stream)), "mec_gemm")
    return O


def _given_workspace(need, workspace, ref):
    """(pointer, bytes) of the workspace: a given one is checked for size and
    device, else one of `need` bytes is allocated."""
    import torch
    if workspace is None:
        workspace = torch.empty(max(need, 1), dtype=torch.uint8, device=ref.device)
    _same_device(workspace, ref, "workspace")
    nbytes = workspace.numel() * workspace.element_size()
    if nbytes < need:
        raise ValueError("the workspace holds %d bytes, %d are needed" % (nbytes, need))
    return workspace, _dev_ptr(workspace, "workspace"), nbytes


def conv2d(I, K, s_h=1, s_w=1, algo="lowered", workspace=None, O=None, stream=None):
    """O = I * K by MEC ("lowered", "fused") or by the im2col baseline
    ("im2col"). With "lowered" or "im2col" a workspace of workspace_bytes(...)
    bytes is allocated unless given (a device tensor of at least that many
    bytes); after the call it holds L (or the im2col matrix). Returns O."""
    d, O = _out(I, K, s_h, s_w, O)
    a = _ALGOS[algo]
    dt = _dtype_code(I)
    ws_ptr, ws_bytes = None, 0
    if a != FUSED:
        need = workspace_bytes(*d, dtype=dt, algo=a)
        workspace, ws_ptr, ws_bytes = _given_workspace(need, workspace, I)
    _check(lib.mec_conv2d(_dev_ptr(I, "I"), _dev_ptr(K, "K"), _dev_ptr(O, "O"), ws_ptr, ws_bytes,
                          *d, dt, a, _stream_handle(stream)), "mec_conv2d")
    return O


# ---------------------------------------------------------------- training passes
# Gradients of the convolution through MEC's lowered layout, fp32 only. G is
# dloss/dO (O's shape, float32).

def grad_workspace_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype=F32,
                         grad_pass=GRAD_INPUT):
    return _check(lib.mec_grad_workspace_bytes(i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w, dtype,
                                               grad_pass), "mec_grad_workspace_bytes")


def _f32(t, name):
    import torch
    if t.dtype != torch.float32:
        raise TypeError("%s must be float32" % name)
    return _dev_ptr(t, name)


def fold(dL, i_w, s_w, dI=None, stream=None):
    """The adjoint of the lowering: dI[n, h, s_w*w + b, c] += dL[n, w, h, b, c]
    for dL of L's shape (i_n x o_w x i_h x k_w x i_c, float32). Returns dI."""
    import torch
    if dL.dim() != 5:
        raise ValueError("dL must be i_n x o_w x i_h x k_w x i_c")
    i_n, o_w, i_h, k_w, i_c = dL.shape
    if output_dims(i_h, i_w, 1, k_w, 1, s_w)[1] != o_w:
        raise ValueError("i_w, k_w, s_w do not give dL's o_w")
    shape = (i_n, i_h, i_w, i_c)
    if dI is None:
        dI = torch.empty(shape, dtype=torch.float32, device=dL.device)
    _check_out(dI, shape, torch.float32, dL, "dI")
    _check(lib.mec_fold(_f32(dL, "dL"), _f32(dI, "dI"), i_n, i_h, i_w, i_c, 1, k_w, 1, 1, s_w,
                        _stream_handle(stream)), "mec_fold")
    return dI


def _grad_dims(G, K, i_h, i_w, s_h, s_w):
    if G.dim() != 4 or K.dim() != 4:
        raise ValueError("G must be i_n x o_h x o_w x k_c and K k_h x k_w x i_c x k_c")
    k_h, k_w, i_c, k_c = K.shape
    i_n = G.shape[0]
    o_h, o_w = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if tuple(G.shape) != (i_n, o_h, o_w, k_c):
        raise ValueError("G must be i_n x o_h x o_w x k_c = %s" % ((i_n, o_h, o_w, k_c),))
    _same_device(K, G, "K")
    return (i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w)


def dgrad_gemm(G, K, i_h, i_w, s_h=1, s_w=1, dL=None, stream=None):
    """dL = dloss/dL (L's shape, float32): G_h K^T added into every slab."""
    import torch
    d = _grad_dims(G, K, i_h, i_w, s_h, s_w)
    shape = (d[0], G.shape[2], i_h, d[5], d[3])
    if dL is None:
        dL = torch.empty(shape, dtype=torch.float32, device=G.device)
    _check_out(dL, shape, torch.float32, G, "dL")
    _check(lib.mec_dgrad_gemm(_f32(G, "G"), _f32(K, "K"), _f32(dL, "dL"), *d, F32,
                              _stream_handle(stream)), "mec_dgrad_gemm")
    return dL


def conv2d_dgrad(G, K, i_h, i_w, s_h=1, s_w=1, dI=None, workspace=None, stream=None):
    """dI = dloss/dI (I's shape, float32); on the dL path the workspace then
    holds dL, on the sub-pixel phase path the last phase's padded G and kernel."""
    import torch
    d = _grad_dims(G, K, i_h, i_w, s_h, s_w)
    shape = (d[0], i_h, i_w, d[3])
    if dI is None:
        dI = torch.empty(shape, dtype=torch.float32, device=G.device)
    _check_out(dI, shape, torch.float32, G, "dI")
    need = grad_workspace_bytes(*d, grad_pass=GRAD_INPUT)
    workspace, wp, wb = _given_workspace(need, workspace, G)
    _check(lib.mec_conv2d_dgrad(_f32(G, "G"), _f32(K, "K"), _f32(dI, "dI"), wp, wb, *d, F32,
                                _stream_handle(stream)), "mec_conv2d_dgrad")
    return dI


def wgrad_gemm(L, G, k_h, i_w, s_h=1, s_w=1, dK=None, workspace=None, stream=None):
    """dK = dloss/dK from a lowered L (i_n x o_w x i_h x k_w x i_c, float32):
    the sum over h of A_h^T G_h. Returns dK (k_h x k_w x i_c x k_c)."""
    import torch
    if L.dim() != 5 or G.dim() != 4:
        raise ValueError("L must be i_n x o_w x i_h x k_w x i_c and G i_n x o_h x o_w x k_c")
    i_n, o_w, i_h, k_w, i_c = L.shape
    k_c = G.shape[3]
    o_h, o_w2 = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if o_w2 != o_w or tuple(G.shape) != (i_n, o_h, o_w, k_c):
        raise ValueError("L and G do not match the shape")
    _same_device(G, L, "G")
    d = (i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w)
    shape = (k_h, k_w, i_c, k_c)
    if dK is None:
        dK = torch.empty(shape, dtype=torch.float32, device=G.device)
    _check_out(dK, shape, torch.float32, G, "dK")
    need = grad_workspace_bytes(*d, grad_pass=GRAD_KERNEL_FROM_L)
    workspace, wp, wb = _given_workspace(need, workspace, G)
    _check(lib.mec_wgrad_gemm(_f32(L, "L"), _f32(G, "G"), _f32(dK, "dK"), wp, wb, *d, F32,
                              _stream_handle(stream)), "mec_wgrad_gemm")
    return dK


def conv2d_wgrad(I, G, k_h, k_w, s_h=1, s_w=1, dK=None, workspace=None, stream=None):
    """dK = dloss/dK from I: the products read the rows of L straight from I
    (no lowered copy is made); the workspace holds the partial sums of the
    reduction's shares (grad_workspace_bytes(..., GRAD_KERNEL))."""
    import torch
    if I.dim() != 4 or G.dim() != 4:
        raise ValueError("I must be i_n x i_h x i_w x i_c and G i_n x o_h x o_w x k_c")
    i_n, i_h, i_w, i_c = I.shape
    k_c = G.shape[3]
    o_h, o_w = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if tuple(G.shape) != (i_n, o_h, o_w, k_c):
        raise ValueError("G must be i_n x o_h x o_w x k_c = %s" % ((i_n, o_h, o_w, k_c),))
    _same_device(G, I, "G")
    d = (i_n, i_h, i_w, i_c, k_h, k_w, k_c, s_h, s_w)
    shape = (k_h, k_w, i_c, k_c)
    if dK is None:
        dK = torch.empty(shape, dtype=torch.float32, device=G.device)
    _check_out(dK, shape, torch.float32, G, "dK")
    need = grad_workspace_bytes(*d, grad_pass=GRAD_KERNEL)
    workspace, wp, wb = _given_workspace(need, workspace, G)
    _check(lib.mec_conv2d_wgrad(_f32(I, "I"), _f32(G, "G"), _f32(dK, "dK"), wp, wb, *d, F32,
                                _stream_handle(stream)), "mec_conv2d_wgrad")
    return dK


def noalloc_scratch_bytes():
    """Bytes of the library's static device scratch (per GPU) that
    conv2d_wgrad_noalloc keeps its partial sums in."""
    return int(lib.mec_noalloc_scratch_bytes())


def conv2d_wgrad_noalloc(I, G, k_h, k_w, s_h=1, s_w=1, dK=None, stream=None):
    """dK = dloss/dK from I, as conv2d_wgrad, with the partial sums in the
    library's static device scratch instead of a workspace: the C call
    allocates nothing (for graph capture and serving loops; the caller passes
    dK). Calls that overlap on one GPU race on the scratch."""
    import torch
    if I.dim() != 4 or G.dim() != 4:
        raise ValueError("I must be i_n x i_h x i_w x i_c and G i_n x o_h x o_w x k_c")
    i_n, i_h, i_w, i_c = I.shape
    k_c = G.shape[3]
    o_h, o_w = output_dims(i_h, i_w, k_h, k_w, s_h, s_w)
    if tuple(G.shape) != (i_n, o_h, o_w, k_c):
        raise ValueError("G must be i_n x o_h x o_w x k_c = %s" % ((i_n, o_h, o_w, k_c),))
    _same_device(G, I, "G")
    shape = (k_h, k_w, i_c, k_c)
    if dK is None:
        dK = torch.empty(shape, dtype=torch.float32, device=G.device)
    _check_out(dK, shape, torch.float32, G, "dK")
    _check(lib.mec_conv2d_wgrad_noalloc(_f32(I, "I"), _f32(G, "G"), _f32(dK, "dK"), i_n, i_h, i_w,
                                        i_c, k_h, k_w, k_c, s_h, s_w, F32, _stream_handle(stream)),
           "mec_conv2d_wgrad_noalloc")
    return dK


# ---------------------------------------------------------------- layer operators
# What stands beside the convolutions in a network, on the same activations and the same K.
# Activations are tensors with the channels last: contiguous, or 2-D (rows x channels) with
# a row pitch, as a slice of a wider tensor's channels has. They, their gradients, K and dK
# are float32 or bfloat16, all the same; bias, gamma, beta, their gradients and the row
# statistics are float32. No size is 0. Given outputs share no memory with each other or with the
# inputs, except where a function says that one may. The *_workspace_bytes functions are functions
# of their arguments alone and remember their values (0.5 us of a call).

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}
_F32 = torch.float32
# the current stream's handle without a Stream object around it (1.8 us of a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = torch.cuda.current_device


def _activations(t, name, c, dtype, device):
    """The row pitch of activations of c channels."""
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.device != device:
        raise ValueError("%s is on %s, the inputs on %s" % (name, t.device, device))
    return _pitch(t, name, c)


def _pitch(t, name, c):
    if t.is_contiguous():
        return c
    if t.dim() == 2 and t.stride(1) == 1 and t.stride(0) >= c:
        return t.stride(0)
    raise ValueError("%s must be contiguous, or rows of contiguous channels" % name)


def _width(n):
    """Sizes past the C interface's int are refused here, the others there."""
    if n > 0x7fffffff:
        raise MecError(_UNSUPPORTED, "a size of %d" % n)


def _channels(t, name):
    """(shape, rows, channels) of activations, and their dtype's code."""
    shape = t.shape
    if len(shape) < 2:
        raise ValueError("%s must have the channels as its last dimension and at least one more" % name)
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    c = shape[-1]
    _width(c)
    return shape, (t.numel() // c if c else 0), c, dt


def _on_device(t, name):
    """Refuses a tensor in host memory; the others are where this one is."""
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)


def _ptr(t):
    """The pointer of a checked tensor, or None."""
    return None if t is None else t.data_ptr()


def _dense(t, shape, dtype, device, name):
    """Checks a dense tensor of exactly this shape, dtype and device."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError("%s must be %s of shape %s, got %s of shape %s"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    if t.device != device:
        raise ValueError("%s is on %s, the inputs on %s" % (name, t.device, device))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _new(t, shape, dtype, ref, name):
    """A given dense output, checked, or a new one."""
    if t is None:
        return ref.new_empty(shape, dtype=dtype)
    _dense(t, shape, dtype, ref.device, name)
    return t


def _act_code(act):
    code = _ACTS.get(act)
    if code is None:
        raise ValueError("act must be one of %s, got %r" % (", ".join(sorted(_ACTS)), act))
    return code


def _launch(name, device, *args):
    """Calls an entry point on that device's current stream, its last argument."""
    index = device.index
    if index != _current_device():
        with torch.cuda.device(index):
            return _launch(name, device, *args)
    status = getattr(lib, name)(*args, _raw_stream(index))
    if status < 0:
        raise MecError(status, name)


def _on(stream, call, ref, *args, **kwargs):
    """The call with `stream` as the current stream, so that what it allocates (outputs,
    workspaces) belongs to that stream too: memory that the caller's stream still uses, or
    uses again once a workspace is dropped, is not handed to it."""
    if stream.device != ref.device:
        raise ValueError("stream is on %s, the inputs on %s" % (stream.device, ref.device))
    with torch.cuda.stream(stream):
        return call(ref, *args, **kwargs)


def _scratch(need, workspace, ref):
    """(workspace, bytes): a given one is checked for size and device, else one is made."""
    if workspace is None:
        return (ref.new_empty(need, dtype=torch.uint8) if need else None), need
    nbytes = workspace.numel() * workspace.element_size()
    if workspace.device != ref.device:
        raise ValueError("workspace is on %s, the inputs on %s" % (workspace.device, ref.device))
    if nbytes < need:
        raise ValueError("the workspace holds %d bytes, %d are needed" % (nbytes, need))
    if not workspace.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return workspace, nbytes


def _matrix(K, dtype, device):
    """(i_c, k_c) of a kernel that acts on pixels: i_c x k_c, or 1 x 1 x i_c x k_c."""
    shape = K.shape
    if len(shape) == 4 and shape[0] == shape[1] == 1:
        shape = shape[2:]
    elif len(shape) != 2:
        raise ValueError("K must be i_c x k_c, or 1 x 1 x i_c x k_c")
    if K.dtype != dtype:
        raise TypeError("K and the activations must have the same dtype")
    if K.device != device:
        raise ValueError("K is on %s, the inputs on %s" % (K.device, device))
    if not K.is_contiguous():
        raise ValueError("K must be contiguous")
    _width(shape[1])
    return shape


def linear(X, K, bias=None, residual=None, act="none", residual_first=False, Y=None, Z=None, workspace=None,
           stream=None):
    """Y = act(X K + bias) + residual, or act(X K + bias + residual) with residual_first, for
    every pixel of X (... x i_c) and K of i_c x k_c (or 1 x 1 x i_c x k_c); act is "none",
    "relu", "silu" or "gelu" (the tanh form). A given Z (Y's shape) receives act's argument,
    for linear_grad. residual may be Y itself. A given workspace holds at least
    linear_workspace_bytes bytes. Returns Y."""
    if stream is not None:
        return _on(stream, linear, X, K, bias, residual, act, residual_first, Y, Z, workspace)
    xs, rows, i_c, dt = _channels(X, "X")
    device, dtype = X.device, X.dtype
    ki, k_c = _matrix(K, dtype, device)
    if ki != i_c:
        raise ValueError("X must have %d channels, got %d" % (ki, i_c))
    x_pitch = _pitch(X, "X", i_c)
    a = _act_code(act)
    shape = xs[:-1] + (k_c,)
    r_pitch = 0
    if bias is not None:
        _dense(bias, (k_c,), _F32, device, "bias")
    if residual is not None:
        if residual.shape != shape:
            raise ValueError("residual must be of shape %s, got %s" % (tuple(shape), tuple(residual.shape)))
        r_pitch = _activations(residual, "residual", k_c, dtype, device)
    y_pitch = k_c
    if Y is None:
        Y = X.new_empty(shape)
    else:
        if Y.shape != shape or Y.dtype != dtype:
            raise ValueError("Y must be %s of shape %s, got %s of shape %s"
                             % (dtype, tuple(shape), Y.dtype, tuple(Y.shape)))
        y_pitch = _activations(Y, "Y", k_c, dtype, device)
    if Z is not None:
        _dense(Z, shape, dtype, device, "Z")
    nbytes = linear_workspace_bytes(rows, i_c, k_c, dt)
    if nbytes:
        workspace, nbytes = _scratch(nbytes, workspace, X)
    _on_device(X, "X")
    _launch("mec_linear", device, X.data_ptr(), K.data_ptr(), _ptr(bias), _ptr(residual), Y.data_ptr(),
            _ptr(Z), rows, i_c, k_c, x_pitch, r_pitch, y_pitch, dt, a, 1 if residual_first else 0,
            _ptr(workspace) if nbytes else None, nbytes)
    return Y


@functools.lru_cache(4096)
def linear_workspace_bytes(rows, i_c, k_c, dtype=F32):
    return _check(lib.mec_linear_workspace_bytes(rows, i_c, k_c, dtype), "mec_linear_workspace_bytes")


@functools.lru_cache(4096)
def linear_grad_workspace_bytes(rows, i_c, k_c, dtype=F32, act=None):
    """For calls with this activation; without one, enough for calls with any."""
    if act is not None:
        return _check(lib.mec_linear_grad_act_workspace_bytes(rows, i_c, k_c, dtype, _act_code(act)),
                      "mec_linear_grad_act_workspace_bytes")
    return _check(lib.mec_linear_grad_workspace_bytes(rows, i_c, k_c, dtype), "mec_linear_grad_workspace_bytes")


def linear_grad(G, X, K, Z=None, act="none", needs=(True, True, True), dZ=None, dX=None, dK=None, dbias=None,
                workspace=None, stream=None):
    """Gradients of linear for G = dloss/dY: (dX, dK, dbias, dZ). Z is what linear left
    (not needed with act "none"); `needs` says which of dX, dK and dbias are wanted, the
    others come back as None (X may be None without dK). dZ, the gradient of act's argument, is G
    itself with act "none"; the residual's gradient is dZ where it was added first, else G.
    dK has K's dtype and shape, dbias is float32; none of the three is computed from dZ as rounded
    to bfloat16. A given workspace holds at least linear_grad_workspace_bytes bytes. dZ may
    be Z's memory, or a dense G's."""
    if stream is not None:
        return _on(stream, linear_grad, G, X, K, Z, act, needs, dZ, dX, dK, dbias, workspace)
    gs, rows, k_c, dt = _channels(G, "G")
    device, dtype = G.device, G.dtype
    i_c, kc = _matrix(K, dtype, device)
    if kc != k_c:
        raise ValueError("G must have %d channels, got %d" % (kc, k_c))
    g_pitch = _pitch(G, "G", k_c)
    a = _act_code(act)
    need_x, need_k, need_b = needs
    x_pitch, shape = i_c, gs[:-1] + (i_c,)
    if X is not None:
        if X.shape != shape:
            raise ValueError("X must be of shape %s, got %s" % (tuple(shape), tuple(X.shape)))
        x_pitch = _activations(X, "X", i_c, dtype, device)
    elif need_k:
        raise ValueError("X is needed for dK")
    if a:
        if Z is None:
            raise ValueError("Z is needed with act %r" % act)
        _dense(Z, gs, dtype, device, "Z")
        dZ = _new(dZ, gs, dtype, G, "dZ")
    else:
        Z, dZ = None, G
    dX = _new(dX, shape, dtype, G, "dX") if need_x else None
    dK = _new(dK, K.shape, dtype, G, "dK") if need_k else None
    dbias = _new(dbias, (k_c,), _F32, G, "dbias") if need_b else None
    nbytes = 0
    if need_x or need_k or need_b:
        workspace, nbytes = _scratch(linear_grad_workspace_bytes(rows, i_c, k_c, dt, act), workspace, G)
    _on_device(G, "G")
    _launch("mec_linear_grad", device, G.data_ptr(), _ptr(X), K.data_ptr(), _ptr(Z), _ptr(dZ) if a else None, _ptr(dX),
            _ptr(dK), _ptr(dbias), _ptr(workspace) if nbytes else None, nbytes, rows, i_c, k_c, g_pitch, x_pitch, dt, a)
    return dX, dK, dbias, dZ


def layer_norm(X, gamma=None, beta=None, eps=1e-5, Y=None, mean=None, rstd=None, stream=None):
    """Layer norm of every pixel's channels, (X - mean) rstd gamma + beta with rstd =
    1 / sqrt(variance + eps). Returns (Y, mean, rstd); mean and rstd (X's shape without the
    channels, float32) are what layer_norm_grad takes. Y may be X itself."""
    if stream is not None:
        return _on(stream, layer_norm, X, gamma, beta, eps, Y, mean, rstd)
    shape, rows, c, dt = _channels(X, "X")
    device, pixels = X.device, shape[:-1]
    x_pitch = y_pitch = _pitch(X, "X", c)
    if gamma is not None:
        _dense(gamma, (c,), _F32, device, "gamma")
    if beta is not None:
        _dense(beta, (c,), _F32, device, "beta")
    if Y is None:
        Y, y_pitch = X.new_empty(shape), c
    elif Y is not X:
        if Y.shape != shape or Y.dtype != X.dtype:
            raise ValueError("Y must be %s of shape %s, got %s of shape %s"
                             % (X.dtype, tuple(shape), Y.dtype, tuple(Y.shape)))
        y_pitch = _activations(Y, "Y", c, X.dtype, device)
    mean = _new(mean, pixels, _F32, X, "mean")
    rstd = _new(rstd, pixels, _F32, X, "rstd")
    _on_device(X, "X")
    _launch("mec_layer_norm", device, X.data_ptr(), _ptr(gamma), _ptr(beta), Y.data_ptr(), mean.data_ptr(),
            rstd.data_ptr(), rows, c, x_pitch, y_pitch, eps, dt)
    return Y, mean, rstd


@functools.lru_cache(4096)
def layer_norm_grad_workspace_bytes(rows, channels, dtype=F32):
    return _check(lib.mec_layer_norm_grad_workspace_bytes(rows, channels, dtype),
                  "mec_layer_norm_grad_workspace_bytes")


def layer_norm_grad(G, X, mean, rstd, gamma=None, needs=(True, True, True), dX=None, dgamma=None, dbeta=None,
                    workspace=None, stream=None):
    """Gradients of layer_norm for G = dloss/dY: (dX, dgamma, dbeta), of which `needs` says
    which are wanted; the others come back as None. A given workspace holds at least
    layer_norm_grad_workspace_bytes bytes."""
    if stream is not None:
        return _on(stream, layer_norm_grad, G, X, mean, rstd, gamma, needs, dX, dgamma, dbeta, workspace)
    shape, rows, c, dt = _channels(X, "X")
    device, dtype, pixels = X.device, X.dtype, shape[:-1]
    x_pitch = _pitch(X, "X", c)
    if G.shape != shape:
        raise ValueError("G must be of shape %s, got %s" % (tuple(shape), tuple(G.shape)))
    g_pitch = _activations(G, "G", c, dtype, device)
    _dense(mean, pixels, _F32, device, "mean")
    _dense(rstd, pixels, _F32, device, "rstd")
    if gamma is not None:
        _dense(gamma, (c,), _F32, device, "gamma")
    dX = _new(dX, shape, dtype, X, "dX") if needs[0] else None
    dgamma = _new(dgamma, (c,), _F32, X, "dgamma") if needs[1] else None
    dbeta = _new(dbeta, (c,), _F32, X, "dbeta") if needs[2] else None
    nbytes = 0
    if needs[1] or needs[2]:
        workspace, nbytes = _scratch(layer_norm_grad_workspace_bytes(rows, c, dt), workspace, X)
    _on_device(X, "X")
    _launch("mec_layer_norm_grad", device, G.data_ptr(), X.data_ptr(), _ptr(gamma), mean.data_ptr(), rstd.data_ptr(),
            _ptr(dX), _ptr(dgamma), _ptr(dbeta), _ptr(workspace) if nbytes else None, nbytes, rows, c, g_pitch, x_pitch, dt)
    return dX, dgamma, dbeta


@functools.lru_cache(4096)
def orthogonalize_workspace_bytes(batch, rows, cols, dtype=F32):
    return _check(lib.mec_orthogonalize_workspace_bytes(batch, rows, cols, dtype),
                  "mec_orthogonalize_workspace_bytes")


def orthogonalize(U, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7, O=None, workspace=None, stream=None):
    """Newton-Schulz orthogonalisation of an update U, as float32 or bfloat16 matrices: one
    (rows x cols) or a stack of them (batch x rows x cols), or one kernel's gradient
    (k_h x k_w x i_c x k_c, taken as the (k_h*k_w*i_c) x k_c matrix) or a stack of those.
    X = U / (|U|_F + eps), then X <- a X + (b A + c A^2) X with A = X X^T, `steps` times.
    Returns O of U's shape; it may be U itself."""
    if stream is not None:
        return _on(stream, orthogonalize, U, steps, coefficients, eps, O, workspace)
    shape = U.shape
    if len(shape) not in (2, 3, 4, 5):
        raise ValueError("U must be a matrix, a kernel's gradient or a stack of either")
    dt = _DTYPES.get(U.dtype)
    if dt is None:
        raise TypeError("U must be float32 or bfloat16, got %s" % U.dtype)
    if not U.is_contiguous():
        raise ValueError("U must be contiguous")
    batch = shape[0] if len(shape) % 2 else 1
    cols = shape[-1]
    rows = U.numel() // (batch * cols) if batch * cols else 0
    for n in (batch, rows, cols):
        _width(n)
    a, b, c = coefficients
    need = orthogonalize_workspace_bytes(batch, rows, cols, dt)
    O = _new(O, shape, U.dtype, U, "O")
    workspace, nbytes = _scratch(need, workspace, U)
    _on_device(U, "U")
    _launch("mec_orthogonalize", U.device, U.data_ptr(), O.data_ptr(), workspace.data_ptr(), nbytes,
            batch, rows, cols, steps, a, b, c, eps, dt)
    return O
