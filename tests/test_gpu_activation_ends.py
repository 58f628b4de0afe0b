"""Minus infinity through the activations of the matrix product and group norm: what the formulas in gpulet.h say."""

import pytest
import torch

from paper_2109_01611_amd import gpulet

from test_gpu_group_norm import ACT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _expect(y, act):
    if act == "relu":
        assert bool((y == 0).all())
    elif act == "none":
        assert bool((y == -float("inf")).all())
    else:
        assert bool(torch.isnan(y).all())     # minus infinity times zero


@pytest.mark.parametrize("act", sorted(ACT))
def test_minus_infinity(act):
    x, w = torch.ones(5, 1, dtype=torch.bfloat16, device=DEV), torch.full((16, 1), -float("inf"), dtype=torch.bfloat16, device=DEV)
    y = torch.zeros(5, 16, device=DEV)
    gpulet.matmul(gpulet.matmul_desc(x, w, None, y, 5, 16, 1, act=ACT[act], out_dtype=gpulet.F32))
    torch.cuda.synchronize()
    _expect(y, act)
    # group norm: by the residual, in one launch and in two
    for hw in (4, 128):
        x = torch.randn(1, hw, hw, 16, device=DEV)
        r, y = torch.full_like(x, -float("inf")), torch.zeros_like(x)
        d = gpulet.group_norm_desc(x, None, None, y, 1, 16, hw, hw, 2, act=ACT[act], residual=r, dtype=gpulet.F32)
        n = gpulet.group_norm_workspace_bytes(d)
        assert (n > 0) == (hw == 128)
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
        gpulet.group_norm(d, ws, n)
        torch.cuda.synchronize()
        _expect(y, act)
