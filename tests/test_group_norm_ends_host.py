"""Group norm without a GPU: maps too large for a launch, and bounds that a variance from sums of squares does not meet."""

import pytest

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
