"""Plans and workspaces of the layer operators' products, on the CPU: no pointer is read and
nothing launched."""
import ctypes

import pytest
import torch

import kernels as kn
import paper_1706_06873_amd as mec
from test_layers import BF16, F32, FAKE, NULL, linear_grad


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
