"""Group norm without a GPU: maps too large for a launch, and bounds that a variance from sums of squares does not meet."""

import numpy as np
import pytest
import torch

import block_reference as ref
import norm_bounds
from paper_2109_01611_amd import gpulet

A = 1 << 41   # stand-in address, never followed


@pytest.mark.parametrize("N,C,HW,shift,fits", [
    (1 << 20, 32, 2048, 0, True), (1 << 21, 32, 2048, 0, False),            # 8 workgroups of 256 threads an image
    (1 << 10, (1 << 21) + 1, 1, 0, True), (1 << 11, (1 << 21) + 1, 1, 0, False),    # 2049 of 1024
    (1 << 21, 1 << 20, 1, 0, False), (1 << 21, 8, 1 << 20, 0, False), (1 << 21, 8, 1, 2, True),
], ids=str)
def test_launches_have_less_than_2_32_threads(N, C, HW, shift, fits):
    d = gpulet.group_norm_desc(A + shift, None, None, A + shift, N, C, 1, HW, 1)
    if fits:
        gpulet.group_norm_workspace_bytes(d)
        return
    for call in (lambda: gpulet.group_norm_workspace_bytes(d), lambda: gpulet.group_norm(d, 256, 1 << 40)):
        with pytest.raises(gpulet.GpuletError) as e:
            call()
        assert e.value.status == gpulet.EINVAL


def _sequential(v):
    return np.cumsum(v.astype(np.float32), dtype=np.float32)[-1]


def _pairwise(v):
    return np.sum(v.astype(np.float32), dtype=np.float32)


@pytest.mark.parametrize("total", [_sequential, _pairwise], ids=["sequential", "pairwise"])
@pytest.mark.parametrize("size", [(2, 9, 9, 64, 8), (1, 64, 64, 320, 32), (1, 150, 150, 64, 1)], ids=str)
def test_bounds_catch_a_variance_from_sums_of_squares(size, total):
    # the data of the GPU test of large means; mean(x^2) - mean^2 in fp32, the mistake planted in the reference
    N, H, W, C, G = size
    g = torch.Generator().manual_seed(5)
    x = torch.randn(N, H, W, C, generator=g) * (0.5 + torch.rand(C, generator=g)) + torch.randn(C, generator=g) + 1000.0
    x = x.numpy()
    want, err = norm_bounds.group_norm(x, None, None, G, 1e-5)
    bound = ref.rounded_bound(want, err, torch.float32, "none")
    ref.assert_within(want, want, bound)
    s = x.reshape(N, H * W, G, C // G)
    got = np.empty(s.shape)
    for n in range(N):
        for k in range(G):
            v = s[n, :, k].reshape(-1)
            m = total(v) / np.float32(v.size)
            var = total(v * v) / np.float32(v.size) - m * m
            got[n, :, k] = (s[n, :, k].astype(np.float64) - m) / np.sqrt(np.float64(max(var, 0)) + 1e-5)
    with pytest.raises(AssertionError):
        ref.assert_within(got.reshape(x.shape), want, bound)
