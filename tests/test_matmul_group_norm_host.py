"""The matrix product and group norm entry points without a GPU: what they refuse, what workspace they ask for, and that the
bounds of the GPU tests would catch a planted mistake (planted in the reference, not in a kernel)."""

import ctypes

import numpy as np
import pytest
import torch

import block_reference as ref
from paper_2109_01611_amd import gpulet

A = 1 << 20   # stand-in addresses, never followed
MM = dict(x=A, w=2 * A, b=None, y=3 * A, M=64, N=64, K=64)
GN = dict(x=A, gamma=None, beta=None, y=2 * A, N=2, C=64, H=8, W=8, groups=8)


def _refused(make, call, size, base, **kw):
    d = make(**dict(base, **kw))
    for f in (lambda: size(d), lambda: call(d, 64 * A, 1 << 30)):
        with pytest.raises(gpulet.GpuletError) as e:
            f()
        assert e.value.status == gpulet.EINVAL, kw


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(w=None), dict(y=None), dict(M=0), dict(N=0), dict(K=-1), dict(M=(1 << 24) + 1),
    dict(N=(1 << 20) + 1, y=1 << 40), dict(K=(1 << 20) + 1), dict(M=1 << 24, N=4096), dict(ldx=63), dict(ldw=63),
    dict(ldy=63), dict(residual=4 * A, ldr=63), dict(ldx=(1 << 20) + 1), dict(ldx=-64), dict(dtype=gpulet.F32),
    dict(dtype=7), dict(out_dtype=gpulet.F16), dict(dtype=gpulet.F16), dict(act=5), dict(act=-1), dict(x=A + 1),
    dict(w=A + 1), dict(b=A + 2), dict(y=3 * A + 2, out_dtype=gpulet.F32), dict(y=A), dict(y=A + 2 * 64 * 63), dict(y=2 * A - 128),
    dict(b=3 * A + 64), dict(residual=3 * A + 64), dict(residual=3 * A, ldr=128),
    dict(ldx=128, y=A + 126, ldy=128), dict(ldx=96, y=A + 128, ldy=96),      # slices that share columns
], ids=str)
def test_matmul_refuses(kw):
    _refused(gpulet.matmul_desc, gpulet.matmul, gpulet.matmul_workspace_bytes, MM, **kw)


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(y=None), dict(N=0), dict(C=0), dict(H=0), dict(W=-3), dict(groups=0), dict(groups=7), dict(groups=128),
    dict(x_ch_stride=63), dict(y_ch_stride=63), dict(r_ch_stride=63), dict(eps=-1e-5), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(dtype=3), dict(act=5), dict(act=-1), dict(x=A + 1), dict(x=A + 2, dtype=gpulet.F32, y=4 * A),
    dict(gamma=4 * A + 2), dict(beta=2 * A), dict(y=A + 128), dict(y=A, y_ch_stride=128), dict(residual=2 * A + 64),
    dict(H=1 << 12, W=1 << 12, y=1 << 40), dict(H=1 << 16, W=1 << 16, y=1 << 40), dict(N=1 << 20, y=1 << 50),
    dict(H=1 << 10, W=1 << 10, x_ch_stride=1 << 10, y=1 << 40),
], ids=str)
def test_group_norm_refuses(kw):
    _refused(gpulet.group_norm_desc, gpulet.group_norm, gpulet.group_norm_workspace_bytes, GN, **kw)


def test_null_descriptors_and_workspaces():
    n = ctypes.c_size_t()
    for name in ("gpulet_matmul", "gpulet_group_norm"):
        assert getattr(gpulet.lib, name)(None, None, 0, None) == gpulet.EINVAL
        assert getattr(gpulet.lib, name + "_workspace_bytes")(None, ctypes.byref(n)) == gpulet.EINVAL
    d = gpulet.matmul_desc(**MM)
    assert gpulet.lib.gpulet_matmul_workspace_bytes(ctypes.byref(d), None) == gpulet.EINVAL
    # misaligned, or over an operand: refused before anything is launched
    for ws, size in ((64 * A + 64, 1 << 20), (3 * A, 256), (A - 256, 1024), (2 * A + 256, 256)):
        with pytest.raises(gpulet.GpuletError) as e:
            gpulet.matmul(d, ws, size)
        assert e.value.status == gpulet.EINVAL


def test_operands_that_only_look_as_if_they_overlapped():
    ok = [dict(ldx=128, y=A + 128, ldy=128),                     # columns 0..63 in, 64..127 out
          dict(x=A + 128, ldx=128, y=A, ldy=128), dict(residual=3 * A), dict(residual=3 * A, ldr=100, ldy=100),
          dict(b=A, x=2 * A, w=2 * A)]                           # inputs may share memory
    for kw in ok:
        gpulet.matmul_workspace_bytes(gpulet.matmul_desc(**dict(MM, **kw)))
    ok = [dict(y=A), dict(residual=2 * A), dict(y=A, residual=A), dict(x_ch_stride=128, y=A + 128, y_ch_stride=128),
          dict(gamma=3 * A, beta=3 * A), dict(residual=A)]
    for kw in ok:
        gpulet.group_norm_workspace_bytes(gpulet.group_norm_desc(**dict(GN, **kw)))


def test_bounds_catch_planted_mistakes():
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((5, 96)).astype(np.float32), rng.standard_normal((7, 96)).astype(np.float32)
    y, err = ref.matmul(x, w, act="gelu")
    bound = ref.rounded_bound(y, err, torch.bfloat16, "gelu")
    ref.assert_within(y, y, bound)
    x2 = x.copy()
    x2[:, 95] = 0.0                                               # the last product of every sum left out
    with pytest.raises(AssertionError):
        ref.assert_within(ref.matmul(x2, w, act="gelu")[0], y, bound)
    g = rng.standard_normal((2, 3, 5, 12)).astype(np.float32) + 3.0
    y, err = ref.group_norm(g, None, None, 4, 0.01)
    bound = ref.rounded_bound(y, err, torch.float32, "none")
    n = 3 * 5 * 3
    with pytest.raises(AssertionError):                           # divided by n - 1 instead of n
        ref.assert_within(y * np.sqrt((n - 1) / n), y, bound)
    with pytest.raises(AssertionError):                           # eps left out
        z, _ = ref.group_norm(g, None, None, 4, 0.0)
        ref.assert_within(z, y, bound)
