"""Plans and workspaces of the layer operators' products, on the CPU: no pointer is read and
nothing launched."""
import ctypes

import pytest
import torch

import kernels as kn
import paper_1706_06873_amd as mec
from test_layers import BF16, F32, NULL, linear, linear_grad


def test_workspaces_by_activation():
    L = mec.lib
    for rows, i_c, k_c in ((7, 5, 6), (700, 33, 65), (50176, 512, 2048), (3, 4096, 4096)):
        sizes = {a: mec.linear_grad_workspace_bytes(rows, i_c, k_c, BF16, a) for a in ("none", "relu", "silu", "gelu")}
        assert sizes["none"] == sizes["relu"] and sizes["silu"] == sizes["gelu"]
        assert sizes["gelu"] >= 2 * rows * k_c  # what rounding dZ leaves over
        assert mec.linear_grad_workspace_bytes(rows, i_c, k_c, BF16) == max(sizes.values())
        for a in sizes:  # fp32 has nothing to hold
            assert mec.linear_grad_workspace_bytes(rows, i_c, k_c, F32, a) == mec.linear_grad_workspace_bytes(rows, i_c, k_c, F32)
    need = mec.linear_grad_workspace_bytes(7, 5, 6, BF16, "gelu")
    assert need > 0 and mec.linear_grad_workspace_bytes(7, 5, 6, BF16, "relu") == 0
    assert linear_grad(dtype=BF16, act=3, wb=need - 1) == -2 and linear_grad(dtype=BF16, act=3, ws=NULL) == -2
    assert linear_grad(dtype=BF16, act=2, ws=ctypes.c_void_p(0x100002)) == -3
    f = L.mec_linear_grad_act_workspace_bytes
    for bad in ((0, 5, 6, 0, 0), (7, 0, 6, 0, 0), (7, 5, 0, 0, 0), (7, 5, 6, 2, 0), (7, 5, 6, 0, 4), (7, 5, 6, 0, -1)):
        assert f(*bad) == -1
    assert f(7, 1 << 21, 6, 0, 0) == -5
    with pytest.raises(ValueError, match="act must be"):
        mec.linear_grad_workspace_bytes(7, 5, 6, BF16, "tanh")


def test_the_binding_asks_for_the_workspace_of_its_activation():
    t = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    G, X, K, Z = t(8, 6), t(8, 5), t(5, 6), t(8, 6)
    small = torch.zeros(8, dtype=torch.uint8)
    with pytest.raises(ValueError, match="workspace holds"):
        mec.linear_grad(G, X, K, Z, "gelu", workspace=small)
    for act in ("none", "relu"):
        with pytest.raises(ValueError, match="device tensor"):
            mec.linear_grad(G, X, K, Z, act, workspace=small)


# outputs and threads of a workgroup, by the kernels' numbers
TILES = {"f32": {0: (32, 32, 1024), 1: (128, 64, 256), 2: (256, 128, 512), 3: (64, 64, 256), 4: (64, 64, 768)},
         "bf16": {0: (32, 32, 1024), 1: (128, 128, 256), 2: (256, 256, 512), 3: (64, 128, 256), 4: (64, 64, 256),
                  5: (64, 64, 256)}}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [kn.XK, kn.XKT])
@pytest.mark.parametrize("rows,width", [(1 << 30, 1), (1 << 30, 16), (1 << 30, 64), ((1 << 30) - 63, 8), (1 << 29, 128),
                                        (1 << 28, 256), (1 << 25, 2048), (1 << 24, 64)])
def test_plans_are_launches_that_a_grid_holds(dtype, layout, rows, width):
    """Fewer than 2^32 threads, for products of many rows as for a stack of many matrices."""
    for K in (1, 16, 64, 1024):
        for M, batch in ((rows, 1), (rows >> 14, 1 << 14)):
            kernel, shares = kn.product_plan(layout, dtype, M, width, K, batch, batch == 1)
            tm, tn, threads = TILES[dtype][kernel]
            blocks = -(-M // tm) * -(-width // tn) * batch * shares
            assert blocks * threads < 1 << 32, (kernel, shares, K, batch)


def test_outputs_that_no_launch_holds_are_refused():
    """2^40 of them, terabytes: nothing is launched, and nothing before it either."""
    big = dict(rows=1 << 30, k_c=1024, xp=5, rp=1024, yp=1024)
    assert linear(**big) == -5 and linear(dtype=BF16, **big) == -5
    assert mec.lib.mec_linear_workspace_bytes(1 << 30, 5, 1024, F32) == -5
    assert linear_grad(rows=1 << 30, i_c=1024, k_c=5, gp=5, xp=1024, wb=1 << 62) == -5


def test_steps_are_paired_only_where_that_was_shown_to_be_precise():
    """Five steps or more of the default coefficients."""
    for batch, rows, cols in ((1, 256, 2304), (23, 2304, 256), (6, 2016, 53), (2, 32, 2160), (4, 200, 400)):
        assert [kn.orth_pairs(batch, rows, cols, n) for n in range(1, 8)] == [False] * 4 + [True] * 3
        for other in ((1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (4.0, -6.0, 2.5), (3.4445, -4.775, 2.03)):
            assert not any(kn.orth_pairs(batch, rows, cols, n, other) for n in range(1, 11))


@pytest.mark.parametrize("odd", [0, 1])
def test_granules_by_dwords_stay_inside_their_row(odd):
    """Rows of more than 8 elements from an odd or even element on: whole dwords, every element of the
    granule, none from outside the row (the small bf16 kernel's rows at odd elements)."""
    for K in (9, 15, 16, 24, 1001, 4096):
        for k in range(0, K - 7, 8):
            got = mec.lib.mec_internal_dword_granule(odd, k)
            wide, single = got & 0xffff, got >> 16
            read = set(range(wide, wide + 8)) | {single}
            assert read >= set(range(k, k + 8)) and min(read) >= 0 and max(read) < K, (K, k, read)
            assert (odd + wide) % 2 == 0


def test_the_fp32_bound_tells_a_lost_product_of_the_split():
    """Values as hi + mid + lo in bf16, products of all parts but one of the six that the kernels take:
    each loss is above the bound that the kernels are held to on 64 products a sum."""
    g = torch.Generator().manual_seed(64)
    a, b = torch.randn(300, 64, generator=g), torch.randn(64, 280, generator=g)

    def split(x):
        hi = x.bfloat16()
        mid = (x - hi.float()).bfloat16()
        return [t.double() for t in (hi, mid, (x - hi.float() - mid.float()).bfloat16())]
    want, A, B = a.double() @ b.double(), split(a), split(b)
    parts = [(0, 0), (1, 0), (0, 1), (1, 1), (2, 0), (0, 2)]
    bound = 6 * 2.0 ** -24 * want.norm()
    error = lambda keep: (sum(A[i] @ B[j] for i, j in keep) - want).norm()  # noqa: E731
    assert error(parts) <= bound / 6
    for lost in parts:
        assert error([p for p in parts if p != lost]) > bound, lost
