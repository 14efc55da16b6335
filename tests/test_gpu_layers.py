"""Layer operators on the GPU against their formulas in 64 bits on the CPU.

Tolerances are bounds by arithmetic, element by element. A sum of n products in fp32, cut off
rather than rounded at worst, is off by at most n 2^-23 times the sum of the products'
magnitudes, in any order; a result rounded to bf16 by another 2^-8 of itself (fp32: 2^-24)."""
import math

import pytest
import torch

import kernels as kn
import paper_1706_06873_amd as mec

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
C0 = math.sqrt(2 / math.pi)


def act64(act, z):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(C0 * (z + 0.044715 * z ** 3)))
    return z


def slope64(act, z):
    if act == "relu":
        return (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    if act == "gelu":
        h = torch.tanh(C0 * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + h) + 0.5 * z * (1 - h * h) * C0 * (1 + 0.134145 * z * z)
    return torch.ones_like(z)


def act_error(act, z, half):
    """|act(z)| off by its own evaluation: e^-t with t off by 2^-22 of itself, and (bf16) the
    hardware's exp2 and reciprocal; below 2^-100 results may be 0."""
    t = z.abs() if act == "silu" else 2 * C0 * (z + 0.044715 * z ** 3).abs()
    rel = (2 + t.clamp(max=200)) * (2.0 ** -18 if half > 1e-6 else 2.0 ** -21)
    return 0 if act in ("none", "relu") else z.abs().clamp(max=1e30) * 2.0 ** -100 + act64(act, z).abs() * rel


def randn(g, *shape):
    return torch.randn(shape, generator=g)


def rows_of(t, gap):
    """t on the GPU, with `gap` elements between its rows."""
    t = t.to(DEV)
    if not gap:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + gap), 7.0, dtype=t.dtype, device=DEV)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def close(got, want, tol, what):
    got = got.detach().cpu().double().reshape(want.shape)
    bad = (got - want).abs() > tol
    assert torch.isfinite(got).all(), what
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / (tol + 1e-300)).max()))


SIZES = [(1, 1, 1), (1, 5, 3), (1, 2048, 1000), (3, 64, 40), (16, 260, 24), (129, 64, 128), (130, 129, 257), (65, 7, 1), (37, 1, 70),
         (300, 1000, 72), (257, 512, 264), (33, 363, 96)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,i_c,k_c", SIZES)
def test_linear(dtype, rows, i_c, k_c):
    acts = ["none", "relu", "silu", "gelu"]
    for n, (gap, res, first, bias) in enumerate([(0, 0, 0, 1), (3, 1, 0, 1), (8, 1, 1, 0), (0, 1, 1, 1)]):
        act = acts[(n + rows) % 4]
        g = torch.Generator().manual_seed(rows * 7 + i_c + n)
        X, K = randn(g, rows, i_c).to(dtype), (randn(g, i_c, k_c) / math.sqrt(i_c)).to(dtype)
        b, R = randn(g, k_c), randn(g, rows, k_c).to(dtype)
        Y = torch.full((rows, k_c + gap), 7.0, dtype=dtype, device=DEV)
        Z = torch.full((rows, k_c), 7.0, dtype=dtype, device=DEV)
        print("[case]", dtype, rows, i_c, k_c, act, gap, res, first, flush=True)
        out = mec.linear(rows_of(X, gap), K.to(DEV), b.to(DEV) if bias else None, rows_of(R, gap) if res else None, act,
                         bool(first), Y=Y[:, :k_c], Z=Z)
        torch.cuda.synchronize()
        assert out.data_ptr() == Y.data_ptr()
        x, k, r = X.double(), K.double(), R.double() * res
        z = x @ k + b.double() * bias + (r if first else 0)
        err = (i_c + 8) * 2.0 ** -23 * (x.abs() @ k.abs() + b.abs().double() * bias + r.abs())
        close(Z, z, err + HALF[dtype] * z.abs(), "Z")
        y = act64(act, z) + (0 if first else r)
        tol = 1.13 * err + act_error(act, z, HALF[dtype]) + 2.0 ** -22 * r.abs()  # |act'| < 1.13
        close(Y[:, :k_c], y, tol + HALF[dtype] * (y.abs() + tol), "Y")
        assert (Y[:, k_c:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,i_c,k_c", SIZES + [(5000, 40, 24), (9001, 33, 130), (4100, 128, 256),
                                                        (2000, 300, 301), (1134, 374, 112), (700, 130, 1001)])
def test_linear_grad(dtype, rows, i_c, k_c):
    for n, (act, gap) in enumerate([("none", 0), ("relu", 3), ("silu", 0), ("gelu", 8)]):
        g = torch.Generator().manual_seed(rows + i_c * 3 + k_c + n)
        X, K = randn(g, rows, i_c).to(dtype), (randn(g, i_c, k_c) / math.sqrt(i_c)).to(dtype)
        G, Z = randn(g, rows, k_c).to(dtype), (2 * randn(g, rows, k_c)).to(dtype)
        print("[case]", dtype, rows, i_c, k_c, act, gap, flush=True)
        Gd = rows_of(G, gap)
        dX, dK, db, dZ = mec.linear_grad(Gd, rows_of(X, gap), K.to(DEV), Z.to(DEV), act)
        torch.cuda.synchronize()
        x, k, q = X.double(), K.double(), G.double()
        dz = q * slope64(act, Z.double())
        # slopes lie within 1.13, their evaluation within 2^-15 (bf16) or 2^-18 (|z| < 12)
        ez = 0 if act in ("none", "relu") else q.abs() * (2.0 ** -15 if dtype is BF16 else 2.0 ** -18)
        if act == "none":
            assert dZ is Gd
        else:
            close(dZ, dz, ez + HALF[dtype] * (dz.abs() + ez), "dZ")
        eb = (rows + 8) * 2.0 ** -23 * dz.abs().sum(0) + (ez.sum(0) if torch.is_tensor(ez) else 0)
        close(db, dz.sum(0), eb, "dbias")
        ez = ez + (0 if act == "none" else HALF[dtype] * dz.abs())  # the products take dZ as rounded
        ez = ez + 0 * dz
        ex = (k_c + 8) * 2.0 ** -23 * (dz.abs() @ k.abs().T) + 1.01 * (ez @ k.abs().T)
        want = dz @ k.T
        close(dX, want, ex + HALF[dtype] * (want.abs() + ex), "dX")
        ek = (rows + 8) * 2.0 ** -23 * (x.abs().T @ dz.abs()) + 1.01 * (x.abs().T @ ez)
        want = x.T @ dz
        close(dK, want, ek + HALF[dtype] * (want.abs() + ek), "dK")


LONG = [(70, 16384, 33), (512, 9000, 64), (1000, 4099, 131), (257, 8192, 72)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,i_c,k_c", LONG)
def test_long_reductions_in_shares(dtype, rows, i_c, k_c):
    """Few outputs of long reductions: the shares' sums lie in the workspace before the epilogue."""
    code = mec.F32 if dtype is F32 else mec.BF16
    if i_c > 8000 or dtype is F32:  # (in bf16 the shortest is not worth the second launch)
        assert mec.linear_workspace_bytes(rows, i_c, k_c, code) >= 2 * rows * k_c * 4
        assert mec.linear_grad_workspace_bytes(rows, k_c, i_c, code) >= 2 * rows * k_c * 4
    test_linear(dtype, rows, i_c, k_c)
    test_linear_grad(dtype, rows, k_c, i_c)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shares_in_place_with_a_workspace_of_the_callers(dtype):
    g = torch.Generator().manual_seed(12)
    X, K, R = (randn(g, *s).to(dtype).to(DEV) for s in ((512, 9000), (9000, 64), (512, 64)))
    need = mec.linear_workspace_bytes(512, 9000, 64, mec.F32 if dtype is F32 else mec.BF16)
    ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device=DEV)
    want = mec.linear(X, K, residual=R, act="gelu")
    got = mec.linear(X, K, residual=R, act="gelu", Y=R, workspace=ws[:need])
    assert got is R and torch.equal(R, want) and (ws[need:] == 0x7f).all()


def test_linear_grad_wants_only_some():
    g = torch.Generator().manual_seed(5)
    X, K, G = randn(g, 70, 24).to(DEV), randn(g, 24, 40).to(DEV), randn(g, 70, 40).to(DEV)
    full = mec.linear_grad(G, X, K)
    for needs in ((True, False, False), (False, True, False), (False, False, True), (False, False, False)):
        some = mec.linear_grad(G, X if needs[1] else None, K, needs=needs)
        for want, a, b in zip(needs, full, some):
            assert torch.equal(a, b) if want else b is None


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_slopes_are_the_activations_differences(act):
    """G = 1 and K = 1x1: dZ is the slope, against differences of the activation in 64 bits
    (step 1e-5: off by 1e-10/6 |act'''| < 1e-9)."""
    z = torch.cat([torch.linspace(-14, 14, 1001), torch.tensor([0.0, -0.0, 1e-30, -90.0, 90.0, 1e20, -1e20])])
    Z = z.reshape(-1, 1).to(DEV)
    dZ = mec.linear_grad(torch.ones_like(Z), Z, torch.ones(1, 1, device=DEV), Z, act)[3]
    zd = z.double()
    zc = zd.clamp(-50, 50)  # the slope is 0 or 1 to 64 bits beyond
    want = (act64(act, zc + 1e-5) - act64(act, zc - 1e-5)) / 2e-5
    want = torch.where(zd.abs() > 50, (zd > 0).double(), want)
    close(dZ[:, 0], want, 1e-8 + 2.0 ** -18 * want.abs() + 2.0 ** -20, act)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,i_c,k_c", [(40, 72, 48), (150, 200, 136), (5, 100, 33)])
def test_linear_spreads_infinities_and_nans_as_the_formula(dtype, rows, i_c, k_c):
    """Other rows and columns are as without them, also where the reduction ends in a tile."""
    g = torch.Generator().manual_seed(9)
    X, K = randn(g, rows, i_c).to(dtype), randn(g, i_c, k_c).to(dtype)
    clean = mec.linear(X.to(DEV), K.to(DEV)).cpu()
    X[1, i_c - 1], X[3, 0], K[2, 4] = math.inf, math.nan, -math.inf
    X[rows - 1, i_c - 1] = math.inf  # behind it lies the end of memory, or nothing
    Y = mec.linear(X.to(DEV), K.to(DEV), act="relu").cpu()
    want = (X.double() @ K.double())
    odd = ~torch.isfinite(want)
    want = torch.where(want < 0, torch.zeros_like(want), want)
    assert torch.equal(torch.isnan(Y), torch.isnan(want))
    assert torch.equal(torch.isinf(Y), torch.isinf(want))
    ok = clean.clamp(min=0)
    assert torch.allclose(Y[~odd].float(), ok[~odd].float(), rtol=2.0 ** -7, atol=1e-4)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_and_paired_products_spread_infinities_and_nans(dtype):
    """The same where workgroups or waves share a reduction, and where two products share a launch."""
    g = torch.Generator().manual_seed(10)

    def check(got, want, size):
        got = got.cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
        ok = torch.isfinite(want)
        tol = size + HALF[dtype] * (want.abs() + size)
        assert ((got.double() - want).abs()[ok] <= tol[ok]).all()

    def product(a, b):  # (finite magnitudes for the bound)
        m = lambda t: torch.nan_to_num(t.double().abs(), 0.0, 0.0, 0.0)  # noqa: E731
        return a.double() @ b.double(), (a.shape[1] + 8) * 2.0 ** -23 * (m(a) @ m(b))

    for rows, i_c, k_c in [(512, 9000, 64), (600, 4100, 1000)]:
        X, K = randn(g, rows, i_c).to(dtype), randn(g, i_c, k_c).to(dtype)
        X[1, i_c - 1], X[3, 0], K[2, 4], X[rows - 1, i_c // 2] = math.inf, math.nan, -math.inf, -math.inf
        print("[case]", dtype, rows, i_c, k_c, flush=True)
        check(mec.linear(X.to(DEV), K.to(DEV)), *product(X, K))
    rows, i_c, k_c = 2000, 296, 304
    X, K, G = randn(g, rows, i_c).to(dtype), randn(g, i_c, k_c).to(dtype), randn(g, rows, k_c).to(dtype)
    X[5, 7], G[70, 300], G[1999, 0] = math.inf, math.nan, -math.inf
    dX, dK, db, _ = mec.linear_grad(G.to(DEV), X.to(DEV), K.to(DEV))
    check(dX, *product(G, K.T))
    check(dK, *product(X.T, G))
    assert torch.isnan(db[300]) and db[0] == -math.inf and torch.isfinite(db[1:300]).all()


def test_linear_far_values_fp32():
    """Values at the ends of fp32's range: what the split into bf16 parts does not hold."""
    g = torch.Generator().manual_seed(10)
    for scale_x, scale_k in ((1e-37, 1.0), (1e-30, 1e30), (3e38, 1e-3), (1e-20, 1e-18)):
        X, K = (randn(g, 70, 48).clamp(-1, 1) * scale_x), (randn(g, 48, 40).clamp(-1, 1) * scale_k)
        Y = mec.linear(X.to(DEV), K.to(DEV))
        x, k = X.double(), K.double()
        close(Y, x @ k, 56 * 2.0 ** -23 * (x.abs() @ k.abs()) + 48 * 2.0 ** -126, (scale_x, scale_k))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [kn.XK, kn.XKT, kn.XTK])
def test_every_product_kernel(dtype, layout):
    """Each kernel on shapes that the calls may give to another: tiles with ragged ends, several
    tiles, one and many chunks, rows with a pitch, and shares of the reduction."""
    for M, N, K, gap, splits in [(300, 280, 200, 0, 1), (257, 264, 64, 8, 1), (130, 67, 77, 3, 1), (5, 9, 700, 0, 1),
                                 (264, 520, 1064, 0, 1), (136, 72, 2000, 0, 7), (33, 200, 517, 5, 3)]:
        g = torch.Generator().manual_seed(M + N + K)
        a, b = randn(g, M, K).to(dtype), randn(g, K, N).to(dtype)
        want = a.double() @ b.double()
        err = (K + 8) * 2.0 ** -23 * (a.double().abs() @ b.double().abs())
        A = rows_of(a.T.contiguous() if layout == kn.XTK else a, gap)
        B = rows_of(b.T.contiguous() if layout == kn.XKT else b, gap)
        ran = 0
        for kernel in range(8):
            if splits > 1 and kernel == 0:
                continue
            print("[case]", dtype, layout, M, N, K, gap, splits, kernel, flush=True)
            Y = kn.product(kernel, layout, A, B, splits)
            if Y is not None:
                close(Y, want, err + HALF[dtype] * (want.abs() + err), kernel)
                ran += 1
        assert ran >= 3


def test_linear_in_place_and_shapes():
    g = torch.Generator().manual_seed(11)
    I, K = randn(g, 2, 5, 7, 24).to(DEV), randn(g, 1, 1, 24, 32).to(DEV)
    R = randn(g, 2, 5, 7, 32).to(DEV)
    want = mec.linear(I, K[0, 0], residual=R, act="relu")
    assert want.shape == (2, 5, 7, 32)
    assert mec.linear(I, K, residual=R, act="relu", Y=R).data_ptr() == R.data_ptr()
    assert torch.equal(R, want)
    # the same as the 1x1 convolution, within the order of the sums
    O = mec.conv2d(I, K)
    assert torch.allclose(mec.linear(I, K), O, rtol=0, atol=24 * 2.0 ** -22 * 24)
    dX, dK, db, dZ = mec.linear_grad(O, I, K)
    assert dX.shape == I.shape and dK.shape == K.shape and db.shape == (32,) and dZ is O


# ---------------------------------------------------------------- layer norm

NORM_SIZES = [(1, 1), (3, 2), (1, 7), (5, 64), (49, 2048), (130, 512), (17, 1000), (33, 1001), (9, 4096), (4, 4097), (3, 16384),
              (2, 16386), (2, 40000), (300, 16), (70, 128), (1030, 24), (2100, 136)]


def depth(c):
    """Additions behind one another in a row's sum."""
    return max(64, c // 1024 + 40)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,c", NORM_SIZES)
def test_layer_norm(dtype, rows, c):
    for gap, shift, params in ((0, 0.0, True), (8, 5.0, True), (3, -300.0, False)):
        g = torch.Generator().manual_seed(rows + c)
        X = (randn(g, rows, c) + shift).to(dtype)
        gamma, beta = 1 + 0.3 * randn(g, c), randn(g, c)
        Y = torch.full((rows, c + gap), 7.0, dtype=dtype, device=DEV)
        print("[case]", dtype, rows, c, gap, shift, flush=True)
        y, mean, rstd = mec.layer_norm(rows_of(X, gap), gamma.to(DEV) if params else None, beta.to(DEV) if params else None,
                                       eps=1e-3, Y=Y[:, :c])
        x = X.double()
        ga, be = (gamma.double(), beta.double()) if params else (torch.ones(c).double(), torch.zeros(c).double())
        mu = x.mean(1, keepdim=True)
        r = 1 / torch.sqrt((x - mu).square().mean(1, keepdim=True) + 1e-3)
        xh = (x - mu) * r
        em = depth(c) * 2.0 ** -24 * x.abs().mean(1, keepdim=True)
        close(mean, mu[:, 0], em[:, 0] + 2.0 ** -23 * mu[:, 0].abs(), "mean")
        # the squares are about a mean off by em; each difference is off by 2^-24 of itself
        er = r * (depth(c) * 2.0 ** -23 + 2 * (em * r) + (em * r) ** 2)
        close(rstd, r[:, 0], er[:, 0], "rstd")
        want = xh * ga + be
        tol = ga.abs() * (em * r + xh.abs() * (er / r + 2.0 ** -22)) + 2.0 ** -22 * (be.abs() + want.abs())
        close(y, want, tol + HALF[dtype] * (want.abs() + tol), "Y")
        assert (Y[:, c:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,c", NORM_SIZES)
def test_layer_norm_grad(dtype, rows, c):
    for gap, params in ((0, True), (8, False), (3, True)):
        g = torch.Generator().manual_seed(rows * 3 + c)
        X, G = (2 * randn(g, rows, c) + 1).to(dtype), randn(g, rows, c).to(dtype)
        gamma = 1 + 0.3 * randn(g, c)
        mean = X.double().mean(1)
        rstd = 1 / torch.sqrt((X.double() - mean[:, None]).square().mean(1) + 1e-3)
        mean, rstd = mean.float(), rstd.float()
        print("[case]", dtype, rows, c, gap, flush=True)
        dX, dg, db = mec.layer_norm_grad(rows_of(G, gap), rows_of(X, gap), mean.to(DEV), rstd.to(DEV),
                                         gamma.to(DEV) if params else None)
        q, ga = G.double(), gamma.double() if params else torch.ones(c).double()
        r = rstd.double()[:, None]
        xh = (X.double() - mean.double()[:, None]) * r
        w = q * ga
        want = r * (w - w.mean(1, keepdim=True) - xh * (w * xh).mean(1, keepdim=True))
        tol = depth(c) * 2.0 ** -22 * r * (w.abs() + w.abs().mean(1, keepdim=True)
                                           + xh.abs() * (w * xh).abs().mean(1, keepdim=True))
        close(dX, want, tol + HALF[dtype] * (want.abs() + tol), "dX")
        close(dg, (q * xh).sum(0), (rows + 8) * 2.0 ** -23 * (q * xh).abs().sum(0), "dgamma")
        close(db, q.sum(0), (rows + 8) * 2.0 ** -23 * q.abs().sum(0), "dbeta")


def test_layer_norm_grad_is_the_difference_quotient():
    """The formula's gradient (checked above) against differences of the norm in 64 bits."""
    g = torch.Generator().manual_seed(3)
    x, q, ga = randn(g, 3, 12).double(), randn(g, 3, 12).double(), 1 + 0.3 * randn(g, 12).double()

    def loss(x):
        d = x - x.mean(1, keepdim=True)
        return (q * (d / torch.sqrt(d.square().mean(1, keepdim=True) + 1e-3) * ga)).sum()
    X, G = x.float().to(DEV), q.float().to(DEV)
    _, mean, rstd = mec.layer_norm(X, eps=1e-3)
    dX = mec.layer_norm_grad(G, X, mean, rstd, ga.float().to(DEV), needs=(True, False, False))[0].cpu()
    for i in range(3):
        for j in range(0, 12, 5):
            e = torch.zeros_like(x)
            e[i, j] = 1e-5
            assert abs(float((loss(x + e) - loss(x - e)) / 2e-5) - float(dX[i, j])) < 1e-4


def test_layer_norm_of_one_channel_constants_and_in_place():
    X = torch.full((5, 32), 3.0, device=DEV)
    Y, mean, rstd = mec.layer_norm(X, eps=1e-4)
    assert (Y == 0).all() and (mean == 3).all() and torch.allclose(rstd, torch.tensor(100.0, device=DEV), rtol=1e-6)
    Y, _, rstd = mec.layer_norm(torch.full((5, 32), 3.0, device=DEV), eps=0.0)  # 0 / 0, as the formula
    assert torch.isnan(Y).all() and torch.isinf(rstd).all()
    X = torch.randn(70, 520, device=DEV)
    want = mec.layer_norm(X)[0]
    assert mec.layer_norm(X, Y=X)[0].data_ptr() == X.data_ptr()
    assert torch.equal(X, want)
    X = torch.randn(40, 96, device=DEV)
    bad = X.clone()
    bad[7, 3], bad[9, 1] = math.nan, math.inf
    a, b = mec.layer_norm(X)[0], mec.layer_norm(bad)[0]
    assert torch.isnan(b[7]).all() and torch.isnan(b[9]).all()
    keep = [i for i in range(40) if i not in (7, 9)]
    assert torch.equal(a[keep], b[keep])


# ---------------------------------------------------------------- orthogonalisation

def orth64(U, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    a, b, c = coefficients
    out = []
    for u in U.double():
        x = u / (u.norm() + eps)
        tall = x.shape[0] > x.shape[1]
        x = x.T if tall else x
        for _ in range(steps):
            A = x @ x.T
            x = a * x + (b * A + c * A @ A) @ x
        out.append(x.T if tall else x)
    return torch.stack(out)


# A step multiplies an error by at most 3.9 (the steepest slope of its polynomial over the
# singular values' range 0 to 1.3), so an error e per step grows to at most 311 e over five. A
# step's own errors are the roundings of three products of matrices of norm at most 1.7 per
# singular direction, weighed by at most |b| + 2|c| + a < 13, below 16 * 2^-22 of |X|_F.
ORTH_TOL = 311 * 16 * 2.0 ** -22


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 9), (1, 27, 64), (1, 363, 96), (3, 64, 64), (2, 65, 33), (1, 576, 130),
                                             (2, 100, 300), (1, 200, 1152), (5, 17, 16), (1, 129, 128)])
def test_orthogonalize(dtype, batch, rows, cols):
    g = torch.Generator().manual_seed(rows + cols)
    U = (1e-3 * (randn(g, batch, rows, cols) + 3 * randn(g, batch, rows, 1) * randn(g, batch, 1, cols))).to(dtype)
    print("[case]", dtype, batch, rows, cols, flush=True)
    Ud = U.to(DEV)
    O = mec.orthogonalize(Ud)
    want = orth64(U)
    got = O.cpu().double()
    for i in range(batch):
        err = (got[i] - want[i]).norm() / want[i].norm()
        assert err <= ORTH_TOL + (HALF[dtype] if dtype is BF16 else 0), (i, float(err))
    assert torch.equal(Ud.cpu(), U)
    assert torch.equal(mec.orthogonalize(Ud, O=Ud), O) and torch.equal(Ud, O)


@pytest.mark.parametrize("batch,rows,cols", [(6, 2016, 53), (2, 32, 2160), (1, 50, 260), (3, 128, 1152), (1, 200, 400)])
@pytest.mark.parametrize("noise", [1.0, 0.3, 0.03])
def test_orthogonalize_as_precise_as_single_steps(batch, rows, cols, noise):
    """Steps taken two at once form the second Gram matrix from two products more of the small
    side, each with the roundings of one: at most twice the error of plain steps in fp32."""
    g = torch.Generator().manual_seed(rows)
    k = max(1, min(rows, cols) // 8)
    U = randn(g, batch, rows, k) @ randn(g, batch, k, cols) / k ** 0.5 * (noise < 1) + noise * randn(g, batch, rows, cols)
    print("[case]", batch, rows, cols, noise, flush=True)
    want = orth64(U)
    a, b, c = 3.4445, -4.7750, 2.0315
    X = U / (U.flatten(1).norm(dim=1).view(-1, 1, 1) + 1e-7)
    X = X.mT.contiguous() if rows > cols else X
    for _ in range(5):
        A = X @ X.mT.contiguous()
        X = a * X + (b * A + c * (A @ A)) @ X
    plain = X.mT if rows > cols else X
    got = mec.orthogonalize(U.to(DEV)).cpu()
    err = lambda x: ((x.double() - want).norm() / want.norm()).item()
    assert err(got) <= max(1e-6, 2 * err(plain)), (err(got), err(plain))


def test_orthogonalize_shapes_scales_and_zeros():
    g = torch.Generator().manual_seed(4)
    dK = randn(g, 3, 3, 16, 24).to(DEV)
    O = mec.orthogonalize(dK)
    assert O.shape == dK.shape
    assert torch.equal(O.view(144, 24), mec.orthogonalize(dK.view(144, 24)))
    stack = torch.stack([dK, torch.zeros_like(dK), 2 * dK])
    S = mec.orthogonalize(stack)
    assert torch.equal(S[0], O) and (S[1] == 0).all()
    # what eps leaves of the scale: |U|_F is about 59
    for scale in (1e-12, 1e-30, 1e30):  # (squares beyond fp32)
        s = mec.orthogonalize(dK * scale, eps=0.0).cpu().double()
        assert ((s - O.cpu().double()).norm() / s.norm()) < 2 * ORTH_TOL
    sv = torch.linalg.svdvals(O.view(144, 24).cpu().double())
    assert sv.min() > 0.6 and sv.max() < 1.3
    one = mec.orthogonalize(dK, steps=1, coefficients=(1.5, -0.5, 0.0)).cpu().double().view(144, 24)
    want = orth64(dK.cpu().view(1, 144, 24), 1, (1.5, -0.5, 0.0))[0]
    assert ((one - want).norm() / want.norm()) < 16 * 2.0 ** -22
    bad = stack.clone()
    bad[1, 0, 0, 0, 0] = math.nan
    B = mec.orthogonalize(bad)
    assert torch.equal(B[0], S[0]) and torch.equal(B[2], S[2]) and torch.isnan(B[1]).all()


# ---------------------------------------------------------------- together

def block(I, p, ws=None):
    """conv -> norm -> linear (gelu) -> linear + residual, and its gradients."""
    O = mec.conv2d(I, p["K0"], algo="fused")
    N, mean, rstd = mec.layer_norm(O, p["gamma"], p["beta"])
    Z = torch.empty(N.shape[:-1] + (p["K1"].shape[1],), device=I.device)
    H = mec.linear(N, p["K1"], p["b1"], act="gelu", Z=Z)
    Y = mec.linear(H, p["K2"], p["b2"], residual=O)
    G = 2 * Y  # loss = sum Y^2
    dH, dK2, db2, _ = mec.linear_grad(G, H, p["K2"])
    dN, dK1, db1, _ = mec.linear_grad(dH, N, p["K1"], Z, "gelu")
    dO, dg, dbeta = mec.layer_norm_grad(dN, O, mean, rstd, p["gamma"])
    dO = dO + G
    dK0 = mec.conv2d_wgrad(I, dO, 3, 3)
    return Y, [dK0, dg, dbeta, dK1, db1, dK2, db2], mec.orthogonalize(dK0)


def make_block(seed):
    g = torch.Generator().manual_seed(seed)
    I = randn(g, 2, 12, 11, 8)
    p = {"K0": randn(g, 3, 3, 8, 32) / 8, "gamma": 1 + 0.2 * randn(g, 32), "beta": 0.2 * randn(g, 32),
         "K1": randn(g, 32, 96) / 6, "b1": 0.1 * randn(g, 96), "K2": randn(g, 96, 32) / 10, "b2": 0.1 * randn(g, 32)}
    return I, p


def test_a_block_and_its_gradients_against_differentiation():
    I, p = make_block(0)
    Y, grads, update = block(I.to(DEV), {k: v.to(DEV) for k, v in p.items()})
    q = {k: v.double().requires_grad_() for k, v in p.items()}
    O = torch.nn.functional.conv2d(I.double().permute(0, 3, 1, 2), q["K0"].permute(3, 2, 0, 1)).permute(0, 2, 3, 1)
    d = O - O.mean(-1, keepdim=True)
    N = d / torch.sqrt(d.square().mean(-1, keepdim=True) + 1e-5) * q["gamma"] + q["beta"]
    W = act64("gelu", N @ q["K1"] + q["b1"]) @ q["K2"] + q["b2"] + O
    W.square().sum().backward()
    # relative to the whole: four products in a row of at most 288 terms, 2^-23 each at worst
    tol = 4 * 300 * 2.0 ** -23
    assert (Y.cpu().double() - W.detach()).norm() / W.detach().norm() < tol
    for name, got in zip(("K0", "gamma", "beta", "K1", "b1", "K2", "b2"), grads):
        want = q[name].grad
        assert (got.cpu().double() - want).norm() / want.norm() < 4 * tol, name
    want = orth64(grads[0].cpu().view(1, 72, 32))[0]
    assert (update.view(72, 32).cpu().double() - want).norm() / want.norm() < ORTH_TOL


def test_block_captured_in_a_graph():
    I, p = make_block(1)
    p = {k: v.to(DEV) for k, v in p.items()}
    buf = I.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(buf, p)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, grads, update = block(buf, p)
    for seed in (2, 3, 4):
        J = make_block(seed)[0].to(DEV)
        want = block(J, p)  # eager work between the replays
        torch.cuda.synchronize()
        buf.copy_(J)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want[0]) and torch.equal(update, want[2])
        for a, b in zip(grads, want[1]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_shared_and_paired_products_captured(dtype):
    """Products in shares, the two of a backward pass in one launch and a stack's update, in a
    graph that is replayed between eager calls of the same on other inputs."""
    g = torch.Generator().manual_seed(13)
    inputs = [[randn(g, *s).to(dtype).to(DEV) for s in ((512, 9000), (9000, 64), (2000, 296), (296, 304), (2000, 304), (3, 700, 160))]
              for _ in range(3)]

    def work(X, K, X2, K2, G, U):
        Z = torch.empty_like(G)
        H = mec.linear(X2, K2, act="gelu", Z=Z)
        return (mec.linear(X, K, act="silu"), H, *mec.linear_grad(G, X2, K2, Z, "gelu"), mec.orthogonalize(U))

    fixed = [t.clone() for t in inputs[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work(*fixed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work(*fixed)
    for given in inputs[::-1]:
        want = work(*given)
        for t, v in zip(fixed, given):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_streams_and_repeatability():
    """The same bits every time, also from two streams at once with workspaces of their own."""
    g = torch.Generator().manual_seed(21)
    X, K = randn(g, 3000, 72).to(DEV), randn(g, 72, 136).to(DEV)
    G = randn(g, 3000, 136).to(DEV)
    U = randn(g, 2, 200, 96).to(DEV)
    want = mec.linear_grad(G, X, K)[:3] + (mec.linear(X, K), mec.orthogonalize(U))
    want += mec.layer_norm(X)
    want += mec.layer_norm_grad(X, X, want[6], want[7])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            o = mec.linear_grad(G, X, K)[:3] + (mec.linear(X, K), mec.orthogonalize(U))
            o += mec.layer_norm(X)
            outs.append(o + mec.layer_norm_grad(X, X, o[6], o[7]))
    o = mec.linear_grad(G, X, K, stream=streams[0])
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(want, o):
            assert torch.equal(a, b)


def test_a_given_stream_owns_what_the_call_allocates():
    """Workspaces and outputs made inside a call on another stream are not memory that the
    caller's stream hands out again meanwhile."""
    g = torch.Generator().manual_seed(22)
    X, K = randn(g, 20000, 128).to(DEV), randn(g, 128, 256).to(DEV)
    G, U = randn(g, 20000, 256).to(DEV), randn(g, 4, 600, 128).to(DEV)
    want = mec.linear_grad(G, X, K)[:3] + (mec.orthogonalize(U), mec.linear(X, K)) + mec.layer_norm(X)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        got = mec.linear_grad(G, X, K, stream=side)[:3] + (mec.orthogonalize(U, stream=side), mec.linear(X, K, stream=side))
        got += mec.layer_norm(X, stream=side)
        busy = [torch.full((1 << 20,), 3.0, device=DEV) for _ in range(40)]  # the caller's stream goes on
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        del busy


def spread(t, pitch):
    """t's rows `pitch` elements apart, in memory of their own."""
    wide = torch.empty(t.shape[0], pitch, dtype=t.dtype, device=DEV)
    wide[:, :t.shape[1]] = t.to(DEV)
    return wide[:, :t.shape[1]]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,c,k_c", [(2100, 24, 40), (2305, 200, 264)])
def test_rows_that_lie_past_32_bits(dtype, rows, c, k_c):
    """The widest pitch: the last rows are more than 2^32 bytes (bf16) or elements' worth of
    bytes on from the first. The same bits as from dense rows, which take the same kernels."""
    g = torch.Generator().manual_seed(rows)
    pitch = 1 << 20
    X, R, K, G = randn(g, rows, c), randn(g, rows, k_c), randn(g, c, k_c) / 5, randn(g, rows, k_c)
    X, R, K, G = (t.to(dtype).to(DEV) for t in (X, R, K, G))
    print("[case]", dtype, rows, c, k_c, flush=True)
    want = mec.linear(X, K, residual=R, act="relu")
    Y = spread(torch.zeros(rows, k_c, dtype=dtype), pitch)
    mec.linear(spread(X, pitch), K, residual=spread(R, pitch), act="relu", Y=Y)
    assert torch.equal(Y, want)
    Z = mec.linear(X, K)
    want = mec.linear_grad(G, X, K, Z=Z, act="silu")
    got = mec.linear_grad(spread(G, pitch), spread(X, pitch), K, Z=Z, act="silu")
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    want = mec.linear_grad(G, X, K, act="none")
    got = mec.linear_grad(spread(G, pitch), spread(X, pitch), K, act="none")
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    want = mec.layer_norm(X)
    Y = spread(torch.zeros(rows, c, dtype=dtype), pitch)
    got = mec.layer_norm(spread(X, pitch), Y=Y)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    H = randn(g, rows, c).to(dtype).to(DEV)
    want = mec.layer_norm_grad(H, X, *got[1:])
    got = mec.layer_norm_grad(spread(H, pitch), spread(X, pitch), *got[1:])
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_stacks_past_32_bits():
    """150 matrices of 7.6 million elements, 4.6 GB: the last comes out as it does alone."""
    g = torch.Generator().manual_seed(31)
    one = randn(g, 3811, 2000).to(DEV)
    stack = torch.zeros(150, 3811, 2000, device=DEV)
    stack[149] = one
    stack[77, :, 5] = 1.0
    got = mec.orthogonalize(stack, steps=2)
    assert not got[0].any() and torch.isfinite(got[149]).all()
    alone = mec.orthogonalize(one, steps=2)
    assert (got[149] - alone).norm() <= 2.0 ** -16 * alone.norm()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_the_suites_block(capsys, dtype):
    import json
    from paper_1706_06873_amd import suite
    assert suite.main(["block", "--layers", "cv12", "--batch", "2", "--dtype", dtype, "--reps", "2", "--warmup", "1"]) == 0
    row = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert row["layer"] == "cv12" and row["dtype"] == dtype and row["wide"] == 4 * row["channels"]
    assert set(row["us"]) == {"norm", "widen", "narrow", "narrow_grad", "widen_grad", "norm_grad", "update"}
    assert all(t > 0 for t in row["us"].values())
