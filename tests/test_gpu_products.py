"""The products of the layer operators, kernel by kernel, and what their sums are made of, on
the GPU against 64 bits on the CPU.

Bounds are by arithmetic: n products added in fp32, cut off rather than rounded at worst, are off
by at most n 2^-23 times the sum of the products' magnitudes, in any order; rounding to bf16 is
monotonic, so a bf16 output lies between the roundings of the two ends of its interval."""
import math

import pytest
import torch

import kernels as kn
import paper_1706_06873_amd as mec
from test_gpu_layers import BF16, C0, DEV, F32, HALF, ORTH_TOL, act64, act_error, close, orth64, randn, rows_of, slope64

pytestmark = pytest.mark.gpu


def within(got, want, err, what, decided=0.0):
    """got (bf16) is a rounding of a value within err of want; for `decided` of the elements at
    least there is only one such (that many the test can decide on: err grows as the number n of
    products, the outputs as its root, so about n^1.5 2^-14 of them it cannot)."""
    lo, hi = (want - err).to(BF16), (want + err).to(BF16)
    got = got.detach().cpu().reshape(want.shape)
    assert (got >= lo).all() and (got <= hi).all(), (what, int(((got < lo) | (got > hi)).sum()), want.numel())
    share = float((lo == hi).double().mean())
    assert share >= decided, (what, share)


def slope_without_cancellation(act, z):
    """act'(z) in 64 bits by s(t) and 1 - s(t) = s(-t), for what the sign of a small slope decides: at
    z = -7.25 the GELU's is -1.35e-15 (s = 1.9e-16, times 1 + z 2u' (1 - s)), where 1 + tanh is 0."""
    t = z if act == "silu" else 2 * C0 * (z + 0.044715 * z ** 3)
    s, q = torch.sigmoid(t), torch.sigmoid(-t)
    return s + z * s * q * (1 if act == "silu" else 2 * C0 * (1 + 0.134145 * z * z))


# ---------------------------------------------------------------- dZ with more bits than bf16

@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,i_c,k_c", [(40, 72, 48), (150, 200, 136), (61, 131, 77), (5, 100, 33), (300, 256, 40),
                                          (128, 1024, 1024), (200, 1001, 1024), (64, 4096, 128)])
def test_gradients_in_bf16_take_dz_before_its_rounding(rows, i_c, k_c, act):
    """dX and dK are the correctly rounded products of dZ to 16 bits, element by element, wherever
    the bound leaves one rounding; products of dZ as rounded to bf16 miss about every third."""
    g = torch.Generator().manual_seed(rows + i_c)
    X, K = randn(g, rows, i_c).to(BF16), (randn(g, i_c, k_c) / math.sqrt(i_c)).to(BF16)
    G, Z = randn(g, rows, k_c).to(BF16), (2 * randn(g, rows, k_c)).to(BF16)
    print("[case]", rows, i_c, k_c, act, flush=True)
    dX, dK, _, dZ = mec.linear_grad(G.to(DEV), X.to(DEV), K.to(DEV), Z.to(DEV), act)
    x, k, q = X.double(), K.double(), G.double()
    dz = q * slope64(act, Z.double())
    # the slope's evaluation, and what is left over of two roundings to bf16
    ez = q.abs() * 2.0 ** -15 + dz.abs() * 2.0 ** -16
    close(dZ, dz, q.abs() * 2.0 ** -15 + HALF[BF16] * (dz.abs() + q.abs() * 2.0 ** -15), "dZ")
    ex = (2 * k_c + 8) * 2.0 ** -23 * (dz.abs() @ k.abs().T) + 1.01 * (ez @ k.abs().T)
    within(dX, dz @ k.T, ex, "dX", 0.5 if k_c <= 300 else 0.0)
    ek = (2 * rows + 8) * 2.0 ** -23 * (x.abs().T @ dz.abs()) + 1.01 * (x.abs().T @ ez)
    within(dK, x.T @ dz, ek, "dK", 0.5 if rows <= 150 else 0.0)


PARTS = [(300, 280, 200, 0, 1), (257, 264, 64, 8, 1), (130, 67, 77, 3, 1), (5, 9, 300, 0, 1), (264, 520, 328, 0, 1),
         (72, 40, 1024, 0, 3), (33, 200, 517, 5, 2), (520, 264, 96, 0, 1)]


def two_parts(dz, gap, order):
    """dZ's two parts in one allocation, the first after the second where order is -1, and the
    bytes from the one to the other."""
    first = dz.to(BF16)
    second = (dz - first.double()).to(BF16)
    both = torch.full((2, dz.shape[0] + 1, dz.shape[1] + gap), 7.0, dtype=BF16, device=DEV)
    at = (0, 1) if order > 0 else (1, 0)
    for i, t in zip(at, (first, second)):
        both[i, :dz.shape[0], :dz.shape[1]] = t.to(DEV)
    view = both[at[0], :dz.shape[0], :dz.shape[1]]
    return view, order * both.stride(0) * 2, first.double() + second.double()


@pytest.mark.parametrize("layout", [kn.XKT, kn.XTK])
def test_every_kernel_on_dz_in_two_parts(layout):
    ran = 0
    for M, N, K, gap, splits in PARTS:
        g = torch.Generator().manual_seed(M + N + K)
        order = 1 if K % 2 else -1
        if layout == kn.XKT:  # dZ is A
            dz, b = randn(g, M, K).double(), randn(g, K, N).to(BF16)
            A, second, a = two_parts(dz, gap, order)
            b, B = b.double(), rows_of(b.T.contiguous(), gap)
        else:
            a, dz = randn(g, M, K).to(BF16), randn(g, K, N).double()
            B, second, b = two_parts(dz, gap, order)
            a, A = a.double(), rows_of(a.T.contiguous(), gap)
        err = (2 * K + 8) * 2.0 ** -23 * 1.01 * (a.abs() @ b.abs())
        for kernel in range(6):
            if splits > 1 and kernel == 0:
                continue
            print("[case]", layout, M, N, K, gap, splits, kernel, flush=True)
            Y = kn.product_with(kernel, layout, A, B, splits, second=second)
            within(Y, a @ b, err, kernel, 0.5 if K < 300 else 0.0)
            ran += 1
    assert ran >= 40


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("rows,i_c,k_c", [(40, 72, 48), (150, 201, 136), (2000, 296, 304), (600, 1100, 1000)])
def test_gradients_in_bf16_spread_infinities_and_nans(rows, i_c, k_c, act):
    """As the formulas do from dZ, whatever its second part: infinities in K and X times dZ of either
    sign, and infinities and NaNs in G."""
    g = torch.Generator().manual_seed(17)
    X, K, G = randn(g, rows, i_c), randn(g, i_c, k_c), randn(g, rows, k_c)
    Z = 2 * randn(g, rows, k_c)
    K[3, 5], K[7, k_c - 1], X[4, 2], X[rows - 1, i_c - 1] = math.inf, -math.inf, -math.inf, math.inf
    G[9, 1], G[11, 30], X[20, 8] = math.inf, math.nan, math.nan
    G[13, 5] = 0.0  # a dZ of 0 times an infinity
    X, K, G, Z = (t.to(BF16) for t in (X, K, G, Z))
    print("[case]", rows, i_c, k_c, act, flush=True)
    dX, dK, _, dZ = (t.cpu() for t in mec.linear_grad(G.to(DEV), X.to(DEV), K.to(DEV), Z.to(DEV), act))
    dz = G.double() * slope_without_cancellation(act, Z.double())
    assert torch.equal(torch.isnan(dZ), torch.isnan(dz)) and torch.equal(torch.isinf(dZ), torch.isinf(dz))
    for got, want in ((dX, dz @ K.double().T), (dK, X.double().T @ dz)):
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isposinf(got), torch.isposinf(want))
        assert torch.equal(torch.isneginf(got), torch.isneginf(want))
        ok = torch.isfinite(want)
        # (finite sums of up to 2000 products of order 1: bf16's half step, and far more than the sums' own error)
        assert ((got.double() - want).abs()[ok] <= HALF[BF16] * want.abs()[ok] + 2.0 ** -6).all()


def test_gradients_in_bf16_do_not_touch_what_lies_behind_the_workspace():
    """The workspace of exactly the size asked for, at every 4-byte alignment."""
    g = torch.Generator().manual_seed(18)
    for rows, i_c, k_c in ((70, 24, 40), (2000, 33, 57), (700, 512, 64)):
        X, K, G, Z = (randn(g, *s).to(BF16).to(DEV) for s in ((rows, i_c), (i_c, k_c), (rows, k_c), (rows, k_c)))
        want = mec.linear_grad(G, X, K, Z, "gelu")
        need = mec.linear_grad_workspace_bytes(rows, i_c, k_c, mec.BF16, "gelu")
        for shift in (0, 4, 8, 12):
            ws = torch.full((need + 80,), 0x7f, dtype=torch.uint8, device=DEV)
            print("[case]", rows, i_c, k_c, shift, flush=True)
            got = mec.linear_grad(G, X, K, Z, "gelu", workspace=ws[shift:shift + need + (-need) % 4][:need])
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert (ws[:shift] == 0x7f).all() and (ws[shift + need:] == 0x7f).all()


def test_gradients_in_bf16_captured_and_in_place():
    """dZ in the memory of Z and of G, and a graph replayed between eager calls of the same."""
    g = torch.Generator().manual_seed(19)
    inputs = [[randn(g, *s).to(BF16).to(DEV) for s in ((300, 72), (72, 136), (300, 136), (300, 136))] for _ in range(3)]
    X, K, G, Z = inputs[0]
    want = mec.linear_grad(G, X, K, Z, "silu")
    z, q = Z.clone(), G.clone()
    got = mec.linear_grad(G, X, K, z, "silu", dZ=z)
    assert got[3] is z and all(torch.equal(a, b) for a, b in zip(got, want))
    got = mec.linear_grad(q, X, K, Z, "silu", dZ=q)
    assert got[3] is q and all(torch.equal(a, b) for a, b in zip(got, want))
    fixed = [t.clone() for t in inputs[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mec.linear_grad(fixed[2], fixed[0], fixed[1], fixed[3], "gelu")
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mec.linear_grad(fixed[2], fixed[0], fixed[1], fixed[3], "gelu")
    for given in inputs[::-1]:
        want = mec.linear_grad(given[2], given[0], given[1], given[3], "gelu")
        for t, v in zip(fixed, given):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


# ---------------------------------------------------------------- as many rows as a call may have

def test_as_many_rows_as_there_may_be():
    """2^30 rows of one channel: more tiles of 64 rows than a launch holds. One product per output,
    so the exact one rounded."""
    rows = 1 << 30
    X = torch.empty(rows, 1, dtype=BF16, device=DEV)
    X[:, 0] = torch.arange(rows, device=DEV, dtype=torch.int32).remainder_(997).to(BF16)
    K = torch.tensor([[1.2421875]], dtype=BF16, device=DEV)
    print("[case] linear", flush=True)
    Y = mec.linear(X, K)
    for i in range(0, rows, rows // 4):
        assert torch.equal(Y[i:i + rows // 4], X[i:i + rows // 4] * K)
    del Y
    print("[case] dX", flush=True)
    dX = mec.linear_grad(X, None, K, needs=(True, False, False))[0]
    for i in range(0, rows, rows // 4):
        assert torch.equal(dX[i:i + rows // 4], X[i:i + rows // 4] * K)


# ---------------------------------------------------------------- orthogonalisation

DEFAULT = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("batch,rows,cols", [(1, 256, 2304), (6, 2016, 53), (2, 32, 2160), (4, 200, 400), (3, 128, 1152)])
@pytest.mark.parametrize("noise", [1.0, 0.3])
def test_any_steps_and_coefficients_are_as_precise_as_plain_steps(batch, rows, cols, noise):
    """At most twice the error of the same steps taken one by one in fp32, whose roundings are as many
    and whose sums are ordered otherwise, and one rounding, 2^-24, for what products in six parts
    leave out. (The norm of the plain steps is taken in 64 bits, as the kernels' is.)"""
    g = torch.Generator().manual_seed(rows + 1)
    k = max(1, min(rows, cols) // 8)
    U = randn(g, batch, rows, k) @ randn(g, batch, k, cols) / k ** 0.5 * (noise < 1) + noise * randn(g, batch, rows, cols)
    X0 = U.mT.contiguous() if rows > cols else U
    for co, steps in ((DEFAULT, 1), (DEFAULT, 2), (DEFAULT, 3), (DEFAULT, 4), (DEFAULT, 5), (DEFAULT, 6), ((1.5, -0.5, 0.0), 2),
                      ((1.5, -0.5, 0.0), 5), ((1.875, -1.25, 0.375), 2), ((2.0, -1.5, 0.5), 4), ((2.0, -1.5, 0.5), 5)):
        a, b, c = co
        X = (X0.double() / (X0.double().flatten(1).norm(dim=1).view(-1, 1, 1) + 1e-7)).float()
        for _ in range(steps):
            A = X @ X.mT.contiguous()
            X = a * X + (b * A + c * (A @ A)) @ X
        plain = X.mT if rows > cols else X
        want = orth64(U, steps, co)
        print("[case]", batch, rows, cols, noise, co, steps, flush=True)
        got = mec.orthogonalize(U.to(DEV), steps=steps, coefficients=co).cpu()
        err = lambda x: ((x.double() - want).norm() / want.norm()).item()  # noqa: E731
        assert err(got) <= 2 * err(plain) + 2.0 ** -24, (co, steps, err(got), err(plain))


# ---------------------------------------------------------------- rows at odd elements

@pytest.mark.parametrize("layout", [kn.XK, kn.XKT, kn.XTK])
@pytest.mark.parametrize("K", [1, 7, 8, 9, 16, 24, 33, 264, 1000, 1001, 3239])
def test_small_kernel_on_rows_at_odd_elements(layout, K):
    """bf16 rows that begin inside a dword, every other or all of them, with NaNs around each."""
    g = torch.Generator().manual_seed(K)
    M, N = 37, 45
    a, b = randn(g, M, K).to(BF16), randn(g, K, N).to(BF16)
    want = a.double() @ b.double()
    err = (K + 8) * 2.0 ** -23 * 1.01 * (a.double().abs() @ b.double().abs())

    def placed(t, left, gap):
        pitch = t.shape[1] + gap
        wide = torch.full((t.shape[0] * pitch + 8,), math.nan, dtype=BF16, device=DEV)
        view = wide.as_strided(t.shape, (pitch, 1), left)
        view.copy_(t.to(DEV))
        return view

    at = a.T.contiguous() if layout == kn.XTK else a
    bt = b.T.contiguous() if layout == kn.XKT else b
    for left in (0, 1, 2, 3):
        for odd in (0, 1):
            gap = 2 + (K + odd) % 2
            print("[case]", layout, K, left, gap, flush=True)
            within(kn.product(0, layout, placed(at, left, gap), placed(bt, 3 - left, gap)), want, err, (left, gap))


# ---------------------------------------------------------------- activations at their ends

@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [7, 8, 300])
def test_slopes_at_infinities_and_nans(dtype, width):
    """The smooth slopes' limits, ReLU's choice, and NaN where Z is one; also that dX, dK and dbias
    follow from the dZ that comes of it."""
    inf, nan = math.inf, math.nan
    z = torch.tensor([inf, -inf, nan, 20.0, -20.0, 1e30, -1e30, 0.0, -0.0])
    rows = z.numel()
    Z = z.view(-1, 1).expand(rows, width).contiguous()
    G = torch.full((rows, width), 1.5)
    limits = {"relu": [1, 0, 0, 1, 0, 1, 0, 0, 0], "silu": [1, 0, nan, 1, 0, 1, 0, 0.5, 0.5], "gelu": [1, 0, nan, 1, 0, 1, 0, 0.5, 0.5]}
    for act, slope in limits.items():
        print("[case]", dtype, width, act, flush=True)
        X, K = torch.ones(rows, 3, dtype=dtype, device=DEV), torch.ones(3, width, dtype=dtype, device=DEV)
        dX, dK, db, dZ = (t.cpu().double() for t in mec.linear_grad(G.to(dtype).to(DEV), X, K, Z.to(dtype).to(DEV), act))
        want = 1.5 * torch.tensor(slope).double()
        # (silu at +-20: e^-20 times 20 is 4.2e-8, and 1 minus that)
        tol = 1.5 * 2.0 ** -24 + 1e-7 + HALF[dtype] * want.abs().nan_to_num(0.0)
        d = dZ - want.view(-1, 1)
        assert torch.equal(torch.isnan(dZ), torch.isnan(want).view(-1, 1).expand(rows, width))
        assert (d.abs().nan_to_num(0.0) <= tol.view(-1, 1)).all()
        assert torch.equal(torch.isnan(dX), torch.isnan(want).view(-1, 1).expand(rows, 3))
        assert torch.isnan(dK).all() == torch.isnan(want).any() and torch.isnan(db).all() == torch.isnan(want).any()
    # ReLU selects: what G is where Z is not above 0 does not matter
    G[1], G[4] = nan, inf
    dX, dK, db, dZ = mec.linear_grad(G.to(dtype).to(DEV), X, K, Z.to(dtype).to(DEV), "relu")
    assert (dZ[1] == 0).all() and (dZ[4] == 0).all() and torch.isfinite(dX).all() and torch.isfinite(dK).all()
    assert torch.isfinite(db).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_activations_at_infinities_and_nans(dtype):
    """The formulas as they are: z s(z) at -infinity is -infinity times 0."""
    inf, nan = math.inf, math.nan
    z = torch.tensor([[inf], [-inf], [nan], [100.0], [-100.0]]).to(dtype).to(DEV)
    one = torch.ones(1, 1, dtype=dtype, device=DEV)
    for act, want in (("none", [inf, -inf, nan, 100, -100]), ("relu", [inf, 0, nan, 100, 0]), ("silu", [inf, nan, nan, 100, 0]),
                      ("gelu", [inf, nan, nan, 100, 0])):
        got = mec.linear(z, one, act=act).cpu().float().flatten()
        assert torch.allclose(got, torch.tensor(want, dtype=torch.float32), rtol=0, atol=1e-30, equal_nan=True), (act, got)


# ---------------------------------------------------------------- epilogues

EPILOGUE = [(300, 280, 96, 0), (257, 131, 64, 5), (130, 67, 77, 3), (520, 264, 40, 8), (65, 300, 128, 1), (33, 24, 200, 0)]


@pytest.mark.parametrize("dtype,kernel", [(F32, i) for i in range(5)] + [(BF16, i) for i in range(6)])
def test_every_kernels_epilogue(dtype, kernel):
    """Bias, activation, residual first or last, Z, and R in Y's place, by every kernel whatever the
    plans give it: ragged ends, unaligned pitches. The bounds are test_linear's."""
    for n, (M, N, K, gap) in enumerate(EPILOGUE):
        g = torch.Generator().manual_seed(M + N + K)
        a, b = randn(g, M, K).to(dtype), (randn(g, K, N) / math.sqrt(K)).to(dtype)
        bias, R = randn(g, N), randn(g, M, N).to(dtype)
        A, B = rows_of(a, gap), rows_of(b, 0)
        x, k, r = a.double(), b.double(), R.double()
        for act, res, first, has_bias, keep in (("none", 1, 1, 1, 1), ("relu", 1, 1, 1, 1), ("silu", 1, 0, 1, 0), ("gelu", 1, 0, 0, 1),
                                                ("gelu", 0, 0, 1, 1), ("silu", 1, 1, 0, 0), ("none", 1, 0, 1, 0)):
            print("[case]", dtype, kernel, M, N, K, gap, act, res, first, flush=True)
            wide = torch.full((M, N + gap), 7.0, dtype=dtype, device=DEV)
            in_place = bool(res) and n % 2 == 1
            if in_place:
                wide[:, :N] = R.to(DEV)
            Y = wide[:, :N]
            got = kn.product_with(kernel, kn.XK, A, B, R=None if not res else Y if in_place else rows_of(R, gap),
                                  bias=bias.to(DEV) if has_bias else None, act=act, res_first=bool(first), Z=bool(keep), Y=Y)
            z = x @ k + bias.double() * has_bias + (r if first and res else 0)
            err = (K + 8) * 2.0 ** -23 * (x.abs() @ k.abs() + bias.abs().double() * has_bias + r.abs() * res)
            if keep:
                close(got[1], z, err + HALF[dtype] * z.abs(), (kernel, act, "Z"))
            y = act64(act, z) + (r if res and not first else 0)
            tol = 1.13 * err + act_error(act, z, HALF[dtype]) + 2.0 ** -22 * r.abs() * res  # |act'| < 1.13
            close(Y, y, tol + HALF[dtype] * (y.abs() + tol), (kernel, act, "Y"))
            assert (wide[:, N:] == 7).all()


# ---------------------------------------------------------------- symmetric products

@pytest.mark.parametrize("kernel", range(5))
@pytest.mark.parametrize("layout", [kn.XKT, kn.XTK])
def test_symmetric_products_and_their_mirror_images(kernel, layout):
    """X X^T of one and of several tiles, ragged, by every fp32 kernel: alpha X X^T + beta R + diag I with
    R symmetric, stacks, and shares of the reduction (which leave the sum alone)."""
    for M, K, batch, splits in ((64, 100, 1, 1), (65, 72, 3, 1), (200, 130, 2, 1), (321, 96, 1, 1), (130, 1000, 1, 3),
                                (200, 700, 2, 2), (256, 64, 2, 1)):
        if splits > 1 and kernel == 0:
            continue
        g = torch.Generator().manual_seed(M + K + batch)
        a = randn(g, batch, M, K)
        R = randn(g, batch, M, M)
        R = R + R.mT
        want, err = a.double() @ a.double().mT, (K + 8) * 2.0 ** -23 * (a.double().abs() @ a.double().abs().mT)
        X = (a if layout == kn.XKT else a.mT.contiguous()).to(DEV)
        X, Rd = (X[0], R[0].to(DEV)) if batch == 1 else (X, R.to(DEV))
        print("[case]", kernel, layout, M, K, batch, splits, flush=True)
        Y = kn.product_with(kernel, layout, X, X, splits, symmetric=True, batch=batch)
        close(Y.reshape(want.shape), want, err + 2.0 ** -23 * want.abs(), (kernel, "plain"))
        if splits == 1:
            Y = kn.product_with(kernel, layout, X, X, symmetric=True, batch=batch, R=Rd, alpha=2.0315, beta=-4.775, diag=3.4445)
            full = 2.0315 * want - 4.775 * R.double() + 3.4445 * torch.eye(M).double()
            tol = 2.04 * err + 2.0 ** -22 * (2.04 * want.abs() + 4.78 * R.double().abs() + 3.5)
            close(Y.reshape(want.shape), full, tol, (kernel, "with R"))


@pytest.mark.parametrize("batch,rows,cols,gram,square", [
    (23, 2304, 256, (4, 1), (3, 1)),    # three groups of waves, and tiles with their mirror images
    (4, 321, 330, (3, 1), (3, 1)),      # ragged
    (8, 150, 4000, (3, 13), (0, 1)),    # shares of several ragged tiles
    (40, 100, 2000, (3, 6), (3, 1)),
    (1, 72, 20000, (4, 27), (0, 1)),    # shares of the three groups' tiles
    (60, 200, 230, (3, 1), (3, 1)),
    (1, 700, 900, (3, 3), (0, 1)),
])
def test_orthogonalize_by_symmetric_products(batch, rows, cols, gram, square):
    """Stacks and single matrices whose Gram matrices and squares are computed by halves."""
    assert kn.orth_plan(batch, rows, cols) == gram and kn.orth_plan(batch, rows, cols, gram=False) == square
    g = torch.Generator().manual_seed(rows * 3 + cols)
    few = min(batch, 4)  # as many different ones; the others are copies of these
    U = 1e-3 * (randn(g, few, rows, cols) + 3 * randn(g, few, rows, 1) * randn(g, few, 1, cols))
    print("[case]", batch, rows, cols, flush=True)
    O = mec.orthogonalize(U[torch.arange(batch) % few].to(DEV)).cpu()
    want = orth64(U)
    for i in range(batch):
        err = (O[i].double() - want[i % few]).norm() / want[i % few].norm()
        assert err <= ORTH_TOL, (i, float(err))


# ---------------------------------------------------------------- fp32: all six products of the split

@pytest.mark.parametrize("layout", [kn.XK, kn.XKT, kn.XTK])
def test_fp32_products_to_fp32s_own_precision(layout):
    """64 products a sum, in four steps that cut off at most 2^-23 of their partial sum, half of it on
    average, and three roundings more (the parts left out, the two sums' sum, the output's place):
    6 times 2^-24 of the whole. Leaving out any of the six products of the parts is more (shown on
    the CPU by test_products.py)."""
    g = torch.Generator().manual_seed(64)
    a, b = randn(g, 300, 64), randn(g, 64, 280)
    want = a.double() @ b.double()
    A = (a.T.contiguous() if layout == kn.XTK else a).to(DEV)
    B = (b.T.contiguous() if layout == kn.XKT else b).to(DEV)
    for kernel in range(5):
        got = kn.product(kernel, layout, A, B).cpu().double()
        assert (got - want).norm() <= 6 * 2.0 ** -24 * want.norm(), kernel


# ---------------------------------------------------------------- dX and dK in one launch

@pytest.mark.parametrize("dtype,rows,i_c,k_c,act,route", [
    ("f32", 1000, 1000, 1000, "none", (2, 1)), ("f32", 2000, 300, 301, "silu", (2, 7)), ("f32", 900, 520, 520, "gelu", (2, 2)),
    ("f32", 1134, 374, 112, "none", (2, 4)), ("f32", 700, 130, 1001, "gelu", (1, 1)), ("f32", 40, 72, 48, "relu", (1, 1)),
    ("bf16", 1200, 520, 1032, "none", (2, 1)), ("bf16", 2000, 296, 304, "gelu", (2, 7)), ("bf16", 900, 520, 520, "none", (2, 1)),
    ("bf16", 900, 520, 520, "silu", (2, 2)), ("bf16", 40, 72, 48, "gelu", (2, 1)), ("bf16", 700, 130, 1001, "gelu", (1, 1)),
    ("bf16", 700, 130, 1001, "none", (1, 1)),
])
def test_gradients_of_two_products_in_one_launch(dtype, rows, i_c, k_c, act, route):
    assert kn.linear_grad_route(rows, i_c, k_c, dtype, act) == route
    dt = F32 if dtype == "f32" else BF16
    g = torch.Generator().manual_seed(rows + k_c)
    X, K = randn(g, rows, i_c).to(dt), (randn(g, i_c, k_c) / math.sqrt(i_c)).to(dt)
    G, Z = randn(g, rows, k_c).to(dt), (2 * randn(g, rows, k_c)).to(dt)
    print("[case]", dtype, rows, i_c, k_c, act, flush=True)
    dX, dK, _, dZ = mec.linear_grad(G.to(DEV), X.to(DEV), K.to(DEV), Z.to(DEV), act)
    x, k = X.double(), K.double()
    dz = G.double() * slope64(act, Z.double())
    two = 2 if dt is BF16 and act in ("silu", "gelu") else 1
    # the slope's evaluation, and (bf16) what is left over of two roundings
    ez = 0 * dz if act in ("none", "relu") else G.double().abs() * (2.0 ** -15 if dt is BF16 else 2.0 ** -18) + dz.abs() * 2.0 ** -16 * (two - 1)
    ez = ez + (2.0 ** -24 * dz.abs() if dt is F32 else 0)
    for got, want, bound, n, what in ((dX, dz @ k.T, dz.abs() @ k.abs().T, k_c, "dX"), (dK, x.T @ dz, x.abs().T @ dz.abs(), rows, "dK")):
        spread = ez @ k.abs().T if what == "dX" else x.abs().T @ ez
        err = (two * n + 8) * 2.0 ** -23 * bound + 1.01 * spread
        close(got, want, err + HALF[dt] * (want.abs() + err), what)
        # and each alone, by its own launch: the same but for the order of the sums
        alone = mec.linear_grad(G.to(DEV), X.to(DEV), K.to(DEV), Z.to(DEV), act, needs=(what == "dX", what == "dK", False))[what == "dK"]
        close(alone, want, err + HALF[dt] * (want.abs() + err), what + " alone")


def test_gradients_on_a_given_stream():
    g = torch.Generator().manual_seed(23)
    for dt in (F32, BF16):
        X, K, G, Z = (randn(g, *s).to(dt).to(DEV) for s in ((3000, 72), (72, 136), (3000, 136), (3000, 136)))
        want = mec.linear_grad(G, X, K, Z, "gelu")
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        got = mec.linear_grad(G, X, K, Z, "gelu", stream=side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("layout", [kn.XKT, kn.XTK])
def test_every_kernel_on_two_parts_and_infinities(layout):
    """Infinities in the operand that dZ is multiplied with, infinities and NaNs in dZ, and dZ of 0: by
    every kernel as the formula has them, the finite sums as before."""
    for M, N, K, gap, splits in PARTS:
        g = torch.Generator().manual_seed(M * 3 + N + K)
        order = -1 if K % 2 else 1
        dz, other = (randn(g, M, K), randn(g, K, N)) if layout == kn.XKT else (randn(g, K, N), randn(g, M, K))
        r, c = dz.shape
        dz[0, c // 2], dz[r - 1, 0], dz[r // 2, 1] = math.inf, math.nan, 0.0
        r, c = other.shape
        other[r - 1, c - 1], other[0, c // 3], other[r // 2, 1] = math.inf, -math.inf, math.nan
        other = other.to(BF16)
        first = dz.to(BF16)
        second = torch.where(torch.isfinite(first), dz - first.float(), torch.zeros(())).to(BF16)
        both = torch.full((2, dz.shape[0], dz.shape[1] + gap), 7.0, dtype=BF16, device=DEV)
        at = (0, 1) if order > 0 else (1, 0)
        both[at[0], :, :dz.shape[1]], both[at[1], :, :dz.shape[1]] = first.to(DEV), second.to(DEV)
        Z, jump = both[at[0], :, :dz.shape[1]], order * both.stride(0) * 2
        placed = rows_of(other.T.contiguous(), gap)
        A, B = (Z, placed) if layout == kn.XKT else (placed, Z)
        product = lambda z, o: z @ o if layout == kn.XKT else o @ z  # noqa: E731
        want = product(first.double(), other.double())
        ok = torch.isfinite(want)
        finite = lambda t: torch.nan_to_num(t.double(), 0.0, 0.0, 0.0)  # noqa: E731
        exact = product(finite(first) + finite(second), finite(other))
        err = (2 * K + 8) * 2.0 ** -23 * 1.01 * product(finite(first).abs(), finite(other).abs())
        for kernel in range(6):
            if splits > 1 and kernel == 0:
                continue
            print("[case]", layout, M, N, K, gap, splits, kernel, flush=True)
            Y = kn.product_with(kernel, layout, A, B, splits, second=jump).cpu()
            for same in (torch.isnan, torch.isposinf, torch.isneginf):
                assert torch.equal(same(Y), same(want)), (kernel, same)
            within(Y[ok], exact[ok], err[ok], kernel)
