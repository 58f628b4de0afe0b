"""Group norm where its arithmetic comes to an end: steps longer than an image, and maps of one pixel."""

import pytest
import torch

import block_reference as ref
import norm_bounds
from paper_2109_01611_amd import gpulet

from test_gpu_group_norm import GUARD, Case, _np

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("which", ["x", "residual", "y"])
@pytest.mark.parametrize("pixels", [1, 2])
def test_pixels_further_apart_than_memory_is_long(which, pixels):
    # One pixel, or two, and a distance between pixels of up to 2^31 bytes: the other pixels of a batch of loads and stores
    # do not exist, and nothing may come of their offsets, which pass 32 bits.
    C, far = 8208, 1 << (29 if pixels == 1 else 15)
    c = Case(21, 1, 1, pixels, C, 1, act="relu", res=True, pad=(0, 0, 0))
    ld = dict(x=C, residual=C, y=C)
    ld[which] = far
    room = torch.full(((pixels - 1) * far + C + 4096,), GUARD, dtype=torch.bfloat16, device=DEV)
    src = dict(x=c.x, residual=c.r, y=c.y)
    for p in range(pixels):
        room[p * far:p * far + C].copy_(src[which][0, 0, p])
    at = {k: v.data_ptr() for k, v in src.items()}
    at[which] = room.data_ptr()
    d = gpulet.group_norm_desc(at["x"], c.gamma, c.beta, at["y"], 1, C, 1, pixels, 1, eps=c.eps, act=gpulet.ACT_RELU,
                               residual=at["residual"], x_ch_stride=ld["x"], r_ch_stride=ld["residual"], y_ch_stride=ld["y"])
    size = gpulet.group_norm_workspace_bytes(d)
    assert size > 0                       # the form of two launches
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    gpulet.group_norm(d, ws, size)
    torch.cuda.synchronize()
    if which == "y":
        for p in range(pixels):
            c.y[0, 0, p].copy_(room[p * far:p * far + C])
            room[p * far:p * far + C] = GUARD
    else:
        for p in range(pixels):
            room[p * far:p * far + C] = GUARD
    assert bool((room == GUARD).all())
    c.check(which)


# ---- everything below: N, H, W, C, groups; the first of each list is held in registers, the others take two launches
FORMS = [(2, 9, 9, 64, 8), (1, 64, 64, 320, 32), (1, 150, 150, 64, 1), (1, 1, 3, 8200, 1)]


def _close(c, what):
    y, err = norm_bounds.group_norm(_np(c.x), None if c.gamma is None else _np(c.gamma), None if c.beta is None else _np(c.beta),
                                    c.G, c.eps, None if c.r is None else _np(c.r), c.act)
    ref.assert_within(_np(c.y), y, ref.rounded_bound(y, err, c.dt, c.act), what)
    c.check_guards()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", FORMS, ids=str)
def test_constant_groups_of_any_size(size, dtype):
    for value in (2e19, -3e30, 1e38, 1e-30):
        c = Case(6, *size, dtype=dtype, act="relu", res=True)
        c.x.fill_(value)
        want = torch.relu(c.beta + c.r.float()).to(c.dt)
        assert torch.equal(c.run(), want), value


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size", FORMS, ids=str)
def test_squared_differences_past_fp32(size, dtype):
    # the variance counts as infinite, whichever form runs
    for scale in (1e20, 1e25):
        c = Case(7, *size, dtype=dtype, act="relu", res=True, scale=scale)
        want = torch.relu(c.beta + c.r.float()).to(c.dt)
        assert torch.equal(c.run(), want), scale


OUTLIERS = FORMS + [(1, 16, 16, 32, 1), (1, 7, 7, 160, 1), (3, 5, 13, 48, 4), (1, 256, 256, 64, 1), (2, 200, 200, 40, 2), (1, 300, 300, 24, 1)]


@pytest.mark.parametrize("size", OUTLIERS, ids=str)
def test_first_values_far_from_the_others(size):
    # Sums of differences from a first value that lies far off: their roundings may not be those of the far value's size
    # times their number.  A 256 x 256 x 64 map in fp32 is summed in pieces of 1024 pixels, whose first 32 have the first values.
    N, H, W, C, G = size
    for every, first in ((H * W, 1), (H * W, 32), (1024, 32), (768, 32), (64, 1)):
        for step in (4, C // G):
            c = Case(8, *size, dtype="f32", scale=0.01)
            px = c.x.reshape(N, H * W, C).clone()
            at = torch.arange(H * W, device=DEV) % every < first
            ch = torch.arange(C, device=DEV) % step == 0
            px[:, at[:, None] & ch[None, :]] = 1234.5678
            c.x.copy_(px.view(N, H, W, C))
            c.run()
            _close(c, (every, first, step))


@pytest.mark.parametrize("size", FORMS[:3], ids=str)
def test_large_means(size):
    # bounds that, at a mean of 1000, an fp32 mean(x^2) - mean^2 does not meet (test_group_norm_ends_host.py)
    for dtype, mean in (("f32", 1000.0), ("f32", -30.0), ("f16", 100.0)):
        c = Case(5, *size, dtype=dtype, mean=mean)
        c.run()
        _close(c, (dtype, mean))


def test_two_at_once_on_two_streams():
    cs = [Case(11 + i, *size, act="silu", res=True) for i, size in enumerate([(3, 64, 64, 320, 32), (2, 200, 200, 64, 4)])]
    want = [c.run().clone() for c in cs]
    descs = [c.desc() for c in cs]
    sizes = [gpulet.group_norm_workspace_bytes(d) for d in descs]
    assert min(sizes) > 0
    spaces = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for n in sizes]
    streams = [torch.cuda.Stream() for _ in cs]
    for c in cs:
        c.y.fill_(GUARD)
    torch.cuda.synchronize()
    for _ in range(10):
        for st, d, ws, n in zip(streams, descs, spaces, sizes):
            gpulet.group_norm(d, ws, n, st.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        assert torch.equal(c.y, w)
        c.check_guards()
