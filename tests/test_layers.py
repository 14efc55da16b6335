"""Layer operators: what their entry points refuse, on the CPU. The C ABI's checks with
pointers that are never read, the binding's with CPU tensors (every check runs before a
device pointer is taken)."""
import ctypes

import pytest
import torch

import kernels as kn
import paper_1706_06873_amd as mec

FAKE, ODD, NULL = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x100001), None
BIG = 1 << 40
F32, BF16 = mec.F32, mec.BF16


def linear(X=FAKE, K=FAKE, bias=FAKE, R=FAKE, Y=FAKE, Z=FAKE, rows=7, i_c=5, k_c=6, xp=5, rp=6, yp=6, dtype=F32, act=1,
           ws=FAKE, wb=BIG):
    return mec.lib.mec_linear(X, K, bias, R, Y, Z, rows, i_c, k_c, xp, rp, yp, dtype, act, 0, ws, wb, NULL)


def linear_grad(G=FAKE, X=FAKE, K=FAKE, Z=FAKE, dZ=FAKE, dX=FAKE, dK=FAKE, db=FAKE, ws=FAKE, wb=BIG, rows=7, i_c=5, k_c=6,
                gp=6, xp=5, dtype=F32, act=1):
    return mec.lib.mec_linear_grad(G, X, K, Z, dZ, dX, dK, db, ws, wb, rows, i_c, k_c, gp, xp, dtype, act, NULL)


def norm(X=FAKE, gamma=FAKE, beta=FAKE, Y=FAKE, mean=FAKE, rstd=FAKE, rows=7, c=5, xp=5, yp=5, eps=1e-5, dtype=F32):
    return mec.lib.mec_layer_norm(X, gamma, beta, Y, mean, rstd, rows, c, xp, yp, eps, dtype, NULL)


def norm_grad(G=FAKE, X=FAKE, gamma=FAKE, mean=FAKE, rstd=FAKE, dX=FAKE, dg=FAKE, db=FAKE, ws=FAKE, wb=BIG, rows=7, c=5,
              gp=5, xp=5, dtype=F32):
    return mec.lib.mec_layer_norm_grad(G, X, gamma, mean, rstd, dX, dg, db, ws, wb, rows, c, gp, xp, dtype, NULL)


def orth(U=FAKE, O=FAKE, ws=FAKE, wb=BIG, batch=2, rows=7, cols=5, steps=5, eps=1e-7, dtype=F32):
    return mec.lib.mec_orthogonalize(U, O, ws, wb, batch, rows, cols, steps, 3.4445, -4.775, 2.0315, eps, dtype, NULL)


@pytest.mark.parametrize("call,kw", [
    (linear, dict(rows=0)), (linear, dict(rows=-1)), (linear, dict(i_c=0)), (linear, dict(k_c=0)),
    (linear, dict(xp=4)), (linear, dict(rp=5)), (linear, dict(yp=5)), (linear, dict(dtype=2)), (linear, dict(act=4)),
    (linear, dict(act=-1)), (linear, dict(X=NULL)), (linear, dict(K=NULL)), (linear, dict(Y=NULL)),
    (linear_grad, dict(rows=0)), (linear_grad, dict(i_c=0)), (linear_grad, dict(k_c=-3)), (linear_grad, dict(gp=5)),
    (linear_grad, dict(xp=4)), (linear_grad, dict(dtype=-1)), (linear_grad, dict(act=9)), (linear_grad, dict(G=NULL)),
    (linear_grad, dict(X=NULL)), (linear_grad, dict(K=NULL)), (linear_grad, dict(Z=NULL)), (linear_grad, dict(dZ=NULL)),
    (norm, dict(rows=0)), (norm, dict(c=0)), (norm, dict(xp=4)), (norm, dict(yp=4)), (norm, dict(dtype=2)),
    (norm, dict(X=NULL)), (norm, dict(Y=NULL)), (norm, dict(eps=-1e-9)), (norm, dict(eps=float("nan"))),
    (norm_grad, dict(rows=0)), (norm_grad, dict(c=0)), (norm_grad, dict(gp=4)), (norm_grad, dict(xp=4)),
    (norm_grad, dict(dtype=2)), (norm_grad, dict(G=NULL)), (norm_grad, dict(X=NULL)), (norm_grad, dict(mean=NULL)),
    (norm_grad, dict(rstd=NULL)),
    (orth, dict(batch=0)), (orth, dict(rows=0)), (orth, dict(cols=0)), (orth, dict(steps=0)), (orth, dict(steps=101)),
    (orth, dict(eps=-1.0)), (orth, dict(eps=float("nan"))), (orth, dict(dtype=2)), (orth, dict(U=NULL)),
    (orth, dict(O=NULL)),
])
def test_invalid_arguments(call, kw):
    assert call(**kw) == -1


@pytest.mark.parametrize("call,kw", [
    (linear, dict(xp=(1 << 20) + 1)), (linear, dict(rows=(1 << 30) + 1)), (linear, dict(k_c=1 << 21, rp=1 << 21, yp=1 << 21)),
    (linear_grad, dict(gp=1 << 21)), (linear_grad, dict(i_c=1 << 21, xp=1 << 21)), (norm, dict(c=1 << 21, xp=1 << 21, yp=1 << 21)),
    (norm_grad, dict(xp=1 << 21)), (orth, dict(batch=65536)), (orth, dict(rows=1 << 21)),
])
def test_beyond_the_kernels_limits(call, kw):
    assert call(**kw) == -5


@pytest.mark.parametrize("call,names", [
    (linear, "X K bias R Y Z ws"), (linear_grad, "G X K Z dZ dX dK db ws"), (norm, "X gamma beta Y mean rstd"),
    (norm_grad, "G X gamma mean rstd dX dg db ws"), (orth, "U O"),
])
def test_alignment(call, names):
    for name in names.split():
        assert call(**{name: ODD}) == -3, name


def test_alignment_of_16_bits():
    two = ctypes.c_void_p(0x100002)  # enough for bf16, not for the fp32 parameters
    assert linear(X=two) == -3 and linear(bias=two, dtype=BF16) == -3
    assert norm(gamma=two, dtype=BF16) == -3 and norm_grad(dg=two, dtype=BF16) == -3
    assert linear_grad(db=two, dtype=BF16) == -3


def test_workspaces():
    assert mec.linear_workspace_bytes(7, 5, 6) == 0  # no partial sums of short reductions
    long = dict(rows=512, i_c=16384, k_c=64, xp=16384, rp=64, yp=64)
    need = mec.linear_workspace_bytes(512, 16384, 64)
    assert need >= 2 * 512 * 64 * 4
    assert linear(wb=need - 1, **long) == -2 and linear(ws=NULL, **long) == -2
    assert linear(ws=ODD, **long) == -3
    need = mec.linear_grad_workspace_bytes(700, 5, 6)
    assert need > 0 and mec.linear_grad_workspace_bytes(7, 5, 6) == 0  # few rows need none
    assert linear_grad(rows=700, wb=need - 1) == -2 and linear_grad(rows=700, ws=NULL) == -2
    need = mec.layer_norm_grad_workspace_bytes(7, 5)
    assert need > 0
    assert norm_grad(wb=need - 1) == -2 and norm_grad(ws=NULL) == -2
    need = mec.orthogonalize_workspace_bytes(2, 7, 5)
    assert orth(wb=need - 1) == -2 and orth(ws=NULL) == -2
    L = mec.lib
    for bad in ((0, 5, 6, 0), (7, 0, 6, 0), (7, 5, 0, 0), (7, 5, 6, 2)):
        assert L.mec_linear_grad_workspace_bytes(*bad) == -1
    assert L.mec_layer_norm_grad_workspace_bytes(7, 0, 0) == -1 and L.mec_layer_norm_grad_workspace_bytes(7, 5, 3) == -1
    assert L.mec_orthogonalize_workspace_bytes(1, 0, 5, 0) == -1 and L.mec_orthogonalize_workspace_bytes(1, 5, 5, 2) == -1
    assert L.mec_linear_grad_workspace_bytes(7, 1 << 21, 6, 0) == -5


# ---------------------------------------------------------------- the binding

@pytest.fixture(autouse=True)
def no_launch(monkeypatch, request):
    if "binding" not in request.node.name:
        return

    def refuse(*a, **k):
        raise AssertionError("a launching entry point was called")
    for name in ("linear", "linear_grad", "layer_norm", "layer_norm_grad", "orthogonalize"):
        monkeypatch.setattr(mec.lib, "mec_" + name, refuse)


def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses_linear_operands():
    X, K = _t(2, 3, 4, 5), _t(5, 6)
    for kw, error, match in [
        (dict(X=_t(2, 3, 4)), ValueError, "channels"), (dict(X=_t(5)), ValueError, "channels"),
        (dict(X=X.double()), TypeError, "float32 or bfloat16"), (dict(X=X.bfloat16()), TypeError, "same dtype"),
        (dict(K=_t(6, 5).t()), ValueError, "K must be contiguous"), (dict(K=_t(4, 6)), ValueError, "X must have"),
        (dict(K=_t(5)), ValueError, "K must be"), (dict(K=_t(3, 1, 5, 6)), ValueError, "K must be"),
        (dict(X=X.permute(1, 0, 2, 3)), ValueError, "contiguous"), (dict(X=_t(1, 5).expand(7, 5)), ValueError, "contiguous"),
        (dict(X=_t(7, 10)[:, ::2]), ValueError, "contiguous"),
        (dict(bias=_t(5)), ValueError, "bias must be"), (dict(bias=_t(6).bfloat16()), ValueError, "bias must be"),
        (dict(residual=_t(2, 3, 4, 5)), ValueError, "residual must be"),
        (dict(residual=_t(2, 3, 4, 6).bfloat16()), TypeError, "residual must be"),
        (dict(Y=_t(2, 3, 4, 5)), ValueError, "Y must be"), (dict(Y=_t(2, 3, 4, 6).double()), ValueError, "Y must be"),
        (dict(Z=_t(24, 6)), ValueError, "Z must be"), (dict(act="tanh"), ValueError, "act must be"),
        (dict(), ValueError, "device tensor"),
    ]:
        with pytest.raises(error, match=match):
            mec.linear(**{**dict(X=X, K=K), **kw})


def test_binding_refuses_linear_gradients():
    G, X, K, Z = _t(8, 6), _t(8, 5), _t(5, 6), _t(8, 6)
    for kw, error, match in [
        (dict(G=_t(8, 5)), ValueError, "G must have"), (dict(X=_t(7, 5)), ValueError, "X must be of shape"),
        (dict(X=_t(8, 6)), ValueError, "X must be of shape"), (dict(X=X.bfloat16()), TypeError, "X must be"),
        (dict(K=K.bfloat16()), TypeError, "same dtype"), (dict(X=None), ValueError, "X is needed"),
        (dict(act="relu"), ValueError, "Z is needed"), (dict(act="relu", Z=_t(8, 5)), ValueError, "Z must be"),
        (dict(act="relu", Z=Z.bfloat16()), ValueError, "Z must be"),
        (dict(act="silu", Z=Z, dZ=_t(7, 6)), ValueError, "dZ must be"), (dict(dX=_t(8, 6)), ValueError, "dX must be"),
        (dict(dK=_t(6, 5)), ValueError, "dK must be"), (dict(dbias=_t(5)), ValueError, "dbias must be"),
        (dict(G=_t(300, 6), X=_t(300, 5), workspace=_t(1, dtype=torch.uint8)), ValueError, "workspace holds"),
        (dict(needs=(True, False, False)), ValueError, "device tensor"),
    ]:
        with pytest.raises(error, match=match):
            mec.linear_grad(**{**dict(G=G, X=X, K=K), **kw})


def test_binding_refuses_norm_operands():
    X, p, s = _t(2, 4, 5), _t(5), _t(2, 4)
    for kw, error, match in [
        (dict(X=X.half()), TypeError, "float32 or bfloat16"), (dict(gamma=_t(4)), ValueError, "gamma must be"),
        (dict(beta=p.double()), ValueError, "beta must be"), (dict(Y=_t(8, 5)), ValueError, "Y must be"),
        (dict(mean=_t(8)), ValueError, "mean must be"), (dict(rstd=s.double()), ValueError, "rstd must be"),
        (dict(), ValueError, "device tensor"),
    ]:
        with pytest.raises(error, match=match):
            mec.layer_norm(**{**dict(X=X), **kw})
    for kw, error, match in [
        (dict(G=_t(8, 5)), ValueError, "G must be"), (dict(G=X.bfloat16()), TypeError, "G must be"),
        (dict(mean=_t(8)), ValueError, "mean must be"), (dict(rstd=s.bfloat16()), ValueError, "rstd must be"),
        (dict(gamma=_t(4)), ValueError, "gamma must be"), (dict(dX=_t(8, 5)), ValueError, "dX must be"),
        (dict(dgamma=_t(4)), ValueError, "dgamma must be"), (dict(dbeta=p.double()), ValueError, "dbeta must be"),
        (dict(workspace=_t(1, dtype=torch.uint8)), ValueError, "workspace holds"),
    ]:
        with pytest.raises(error, match=match):
            mec.layer_norm_grad(**{**dict(G=X, X=X, mean=s, rstd=s), **kw})


def test_binding_refuses_updates():
    for U, error, match in [
        (_t(5), ValueError, "U must be"), (_t(1, 1, 1, 1, 1, 1), ValueError, "U must be"),
        (_t(4, 4).double(), TypeError, "float32 or bfloat16"), (_t(4, 4), ValueError, "device tensor"),
        (_t(4, 4).t()[:, :3], ValueError, "device tensor|contiguous"),
    ]:
        with pytest.raises(error, match=match):
            mec.orthogonalize(U)
    with pytest.raises(ValueError, match="O must be"):
        mec.orthogonalize(_t(4, 4), O=_t(16))
    with pytest.raises(ValueError, match="workspace holds"):
        mec.orthogonalize(_t(4, 4), workspace=_t(8, dtype=torch.uint8))
    with pytest.raises(mec.MecError):
        mec.orthogonalize(_t(0, 4))


def test_binding_refuses_sizes_past_the_interfaces_int():
    big = 1 << 32  # would arrive as 0, and 5 more as 5
    meta = lambda *shape: torch.empty(shape, device="meta")
    for call in (lambda: mec.linear(meta(2, big + 5), meta(big + 5, 4)), lambda: mec.linear(meta(2, 4), meta(4, big + 5)),
                 lambda: mec.linear_grad(meta(2, big + 5), meta(2, 4), meta(4, big + 5)), lambda: mec.layer_norm(meta(2, big + 5)),
                 lambda: mec.orthogonalize(meta(big + 5, 2)), lambda: mec.orthogonalize(meta(2, big + 5)),
                 lambda: mec.orthogonalize(meta(big + 5, 2, 2))):
        with pytest.raises(mec.MecError) as e:
            call()
        assert e.value.status == -5


# ---------------------------------------------------------------- which kernel a product takes

@pytest.mark.parametrize("layout,dtype,M,N,K,batch,split,want", [
    (kn.XK, "bf16", 1, 1000, 2048, 1, False, (0, 1)),          # few outputs: the waves share the reduction
    (kn.XK, "f32", 333, 131, 363, 1, False, (0, 1)),
    (kn.XK, "bf16", 16384, 4096, 4096, 1, False, (2, 1)),      # 256 x 256 tiles
    (kn.XK, "f32", 16384, 4096, 1024, 1, False, (2, 1)),       # 256 x 128
    (kn.XK, "f32", 100352, 256, 64, 1, False, (1, 1)),         # short reductions: tiles that overlap
    (kn.XKT, "bf16", 1024, 1024, 1024, 1, False, (5, 1)),      # 64 x 64, a tile per compute unit
])
def test_product_plans(layout, dtype, M, N, K, batch, split, want):
    assert kn.product_plan(layout, dtype, M, N, K, batch, split) == want


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_product_plans_share_long_reductions(dtype):
    kernel, shares = kn.product_plan(kn.XTK, dtype, 512, 2048, 50176, 1, True)
    assert kernel > 0 and 4 <= shares <= 64
    assert kn.product_plan(kn.XTK, dtype, 512, 2048, 50176, 1, False)[1] == 1
    for M, N, K in ((1, 1, 1), (7, 3, 1 << 20), (64, 64, 100000), (1 << 20, 1, 3), (4096, 4096, 131072), (200, 100, 1000)):
        kernel, shares = kn.product_plan(kn.XTK, dtype, M, N, K, 1, True)
        runs = -(-K // 64)
        assert 1 <= shares <= max(1, runs // 4) and (shares - 1) * (-(-runs // shares)) < runs  # none empty
        assert shares * M * N <= max(M * N, 1 << 26)


def test_the_suites_block_layers():
    from paper_1706_06873_amd import suite
    layers = suite.block_layers()
    assert "cv12" in layers and "cv1" not in layers and len(layers) >= 5
