"""Group norm with residual and activation against 64 bits: one value to large maps, odd channel counts, slices, every type,
large means, constant groups, special values, in-place calls, gpu-lets and graphs."""

import numpy as np
import pytest
import torch

import block_reference as ref
from paper_2109_01611_amd import gpulet

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, gpulet.BF16), "f16": (torch.float16, gpulet.F16), "f32": (torch.float32, gpulet.F32)}
ACT = {"none": gpulet.ACT_NONE, "relu": gpulet.ACT_RELU, "silu": gpulet.ACT_SILU, "gelu": gpulet.ACT_GELU,
       "gelu_tanh": gpulet.ACT_GELU_TANH}
GUARD = -768.0


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Case:
    def __init__(self, seed, N, H, W, C, G, dtype="bf16", act="none", affine=True, res=False, pad=(0, 0, 0), shift=0, eps=1e-5,
                 mean=0.0, scale=1.0):
        self.shape, self.G, self.act, self.eps = (N, H, W, C), G, act, eps
        self.dt, self.code = TYPES[dtype]
        g = torch.Generator().manual_seed(seed)

        def place(t, ld):
            flat = torch.full((N * H * W * ld + shift,), GUARD, dtype=self.dt, device=DEV)
            view = flat[shift:].view(N, H, W, ld)[..., :C]
            view.copy_(t.to(DEV).to(self.dt))
            return flat, view
        self.ld = tuple(C + p for p in pad)
        x = torch.randn(N, H, W, C, generator=g) * scale * (0.5 + torch.rand(C, generator=g)) + torch.randn(C, generator=g) * scale + mean
        self.xf, self.x = place(x, self.ld[0])
        self.gamma = (1 + 0.3 * torch.randn(C, generator=g)).to(DEV) if affine else None
        self.beta = (0.3 * torch.randn(C, generator=g)).to(DEV) if affine else None
        self.rf, self.r = place(torch.randn(N, H, W, C, generator=g), self.ld[1]) if res else (None, None)
        self.yf, self.y = place(torch.full((N, H, W, C), GUARD), self.ld[2])

    def desc(self, **kw):
        N, H, W, C = self.shape
        a = dict(x=self.x.data_ptr(), gamma=self.gamma, beta=self.beta, y=self.y.data_ptr(), N=N, C=C, H=H, W=W, groups=self.G,
                 eps=self.eps, act=ACT[self.act], residual=None if self.r is None else self.r.data_ptr(), x_ch_stride=self.ld[0],
                 r_ch_stride=self.ld[1], y_ch_stride=self.ld[2], dtype=self.code)
        a.update(kw)
        return gpulet.group_norm_desc(**a)

    def run(self, stream=None):
        d = self.desc()
        size = gpulet.group_norm_workspace_bytes(d)
        ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None
        torch.cuda.synchronize()
        gpulet.group_norm(d, ws, size, stream)
        torch.cuda.synchronize()
        return self.y

    def check(self, what="", x=None, r=None):
        y, err = ref.group_norm(_np(self.x) if x is None else x, None if self.gamma is None else _np(self.gamma),
                                None if self.beta is None else _np(self.beta), self.G, self.eps,
                                (None if self.r is None else _np(self.r)) if r is None else r, self.act)
        ref.assert_within(_np(self.y), y, ref.rounded_bound(y, err, self.dt, self.act), what)
        self.check_guards()

    def check_guards(self):
        N, H, W, C = self.shape
        flat = self.yf.clone()
        flat[flat.numel() - N * H * W * self.ld[2]:].view(N, H, W, self.ld[2])[..., :C] = GUARD
        assert bool((flat == GUARD).all())


# N, H, W, C, groups
SIZES = [(1, 1, 1, 8, 8), (1, 1, 1, 64, 1), (3, 1, 1, 320, 32), (1, 1, 2, 6, 3), (2, 3, 5, 12, 4), (1, 7, 7, 2048, 32), (2, 8, 8, 1280, 32),
         (1, 8, 8, 30, 30), (5, 9, 11, 96, 32), (1, 16, 16, 640, 32), (1, 5, 3, 41, 1), (2, 37, 29, 82, 2), (3, 14, 14, 1024, 32),
         (1, 64, 64, 320, 32), (2, 56, 56, 64, 32), (1, 33, 31, 960, 32), (1, 64, 64, 24, 1), (1, 100, 100, 16, 16), (2, 50, 60, 136, 8),
         (1, 128, 128, 128, 32), (2, 20, 17, 1031, 1), (1, 3, 300, 8208, 1), (1, 13, 17, 1536, 1), (1, 1, 4000, 48, 2), (40, 4, 4, 72, 8), (1, 200, 210, 33, 3), (1, 96, 96, 512, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_sizes(size, dtype):
    c = Case(1, *size, dtype=dtype)
    c.run()
    c.check()
    c = Case(2, *size, dtype=dtype, act="silu", res=True)
    c.run()
    c.check("residual")


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_activations_with_and_without_scale(act, dtype):
    for affine in (True, False):
        for size in ((2, 6, 6, 80, 8), (1, 40, 40, 320, 32)):
            c = Case(3, *size, dtype=dtype, act=act, affine=affine, res=True)
            c.run()
            c.check((affine, size))
    c = Case(3, 2, 6, 6, 80, 8, dtype=dtype, act=act)
    c.beta = None
    c.run()
    c.check("gamma only")
    c = Case(3, 2, 6, 6, 80, 8, dtype=dtype, act=act)
    c.gamma = None
    c.run()
    c.check("beta only")


@pytest.mark.parametrize("pad", [(320, 0, 0), (0, 8, 16), (1, 0, 0), (0, 3, 0), (0, 0, 5), (2, 4, 6)], ids=str)
def test_channel_slices(pad):
    for size in ((2, 8, 8, 320, 32), (1, 70, 70, 96, 8), (3, 5, 5, 18, 3), (1, 120, 120, 320, 4)):
        for shift in (0, 1, 4):
            for dtype in ("bf16", "f32"):
                c = Case(4, *size, dtype=dtype, act="relu", res=True, pad=pad, shift=shift)
                c.run()
                c.check((size, shift, dtype))


def test_large_means_keep_the_variance():
    # mean 1000 standard deviations away: mean(x^2) - mean^2 in fp32 would be wrong in its first digit
    for size in ((2, 9, 9, 64, 8), (1, 64, 64, 320, 32), (1, 150, 150, 64, 1)):
        c = Case(5, *size, dtype="f32", mean=1000.0)
        c.run()
        c.check(size)


def test_constant_groups():
    for size in ((1, 4, 4, 64, 8), (1, 3, 9, 30, 3), (2, 7, 5, 24, 8), (1, 90, 90, 64, 2), (1, 1, 3, 8200, 1)):
        c = Case(6, *size, act="relu", res=True)
        c.x.fill_(3.3)
        want = torch.relu(c.beta + c.r.float()).to(torch.bfloat16)
        assert torch.equal(c.run(), want), size
        c = Case(6, *size, eps=0.0)
        c.x[..., :size[3] // size[4]] = 3.3
        y = c.run()
        cg = size[3] // size[4]
        assert bool(torch.isnan(y[..., :cg]).all()) and bool(torch.isfinite(y[..., cg:]).all())


@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_special_values_stay_in_their_group_and_image(value):
    for size in ((3, 6, 5, 64, 8), (2, 64, 64, 320, 32), (2, 160, 160, 64, 4)):
        N, H, W, C, G = size
        c = Case(7, *size, act="silu")
        c.x[1, H - 1, W - 1, C - 1] = value
        y = c.run().clone()
        cg = C // G
        assert bool(torch.isnan(y[1, :, :, C - cg:]).all())
        y[1, :, :, C - cg:] = 0
        assert bool(torch.isfinite(y).all())


def test_in_place():
    for size in ((2, 8, 8, 320, 32), (1, 64, 64, 320, 32), (1, 256, 256, 128, 32), (4, 37, 29, 82, 2)):
        a = Case(8, *size, act="silu", res=True)
        want = a.run().clone()
        b = Case(8, *size, act="silu", res=True)
        b.y, b.yf = b.x, b.xf
        assert torch.equal(b.run(), want)
        b = Case(8, *size, act="silu", res=True)
        b.y, b.yf = b.r, b.rf
        assert torch.equal(b.run(), want)


def test_an_image_does_not_depend_on_its_batch_or_gpu_let():
    for size in ((5, 8, 8, 1280, 32), (9, 64, 64, 320, 32), (6, 128, 128, 64, 8), (3, 37, 29, 82, 2)):
        c = Case(9, *size, act="gelu", dtype="f16")
        all_ = c.run().clone()
        one = Case(9, 1, *size[1:], act="gelu", dtype="f16")
        one.gamma, one.beta = c.gamma, c.beta
        for i in range(size[0]):
            one.x.copy_(c.x[i:i + 1])
            assert torch.equal(one.run()[0], all_[i]), (size, i)
        with gpulet.Partition(0, 25, 0) as part:
            c.y.fill_(GUARD)
            assert torch.equal(c.run(part.stream), all_), size


def test_workspace_too_small():
    for size in ((1, 4, 4, 64, 8), (1, 512, 512, 64, 2), (8, 256, 256, 128, 32)):
        c = Case(10, *size)
        d = c.desc()
        need = gpulet.group_norm_workspace_bytes(d)
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=DEV)
            for ws_, n in ((None, 0), (None, need), (ws, need - 1)):
                with pytest.raises(gpulet.GpuletError) as e:
                    gpulet.group_norm(d, ws_, n)
                assert e.value.status == gpulet.ENOMEM


def test_images_past_32_bits():
    # 40 images of 64 MB in fp32: the last ones start beyond 2^31 bytes
    N, H, W, C, G = 40, 128, 128, 1024, 32
    x = torch.randn(N, H, W, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    y = torch.empty_like(x)
    d = gpulet.group_norm_desc(x, None, None, y, N, C, H, W, G, dtype=gpulet.F32)
    size = gpulet.group_norm_workspace_bytes(d)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device=DEV)
    gpulet.group_norm(d, ws, size)
    torch.cuda.synchronize()
    for n in (0, 31, 32, 39):
        want, err = ref.group_norm(_np(x[n:n + 1]), None, None, G, 1e-5)
        ref.assert_within(_np(y[n:n + 1]), want, ref.rounded_bound(want, err, torch.float32, "none"), n)


def test_graphs():
    for size in ((1, 8, 8, 320, 32), (2, 64, 64, 320, 32), (4, 200, 200, 128, 32)):
        c = Case(11, *size, act="silu", res=True)
        want = c.run().clone()
        d = c.desc()
        n = gpulet.group_norm_workspace_bytes(d)
        graphs, keep = [], []
        for _ in range(2):
            ws = torch.full((max(n, 1),), 0xFF, dtype=torch.uint8, device=DEV)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                gpulet.group_norm(d, ws, n, torch.cuda.current_stream().cuda_stream)
            graphs.append(g)
            keep.append(ws)
        for i in range(4):
            c.y.fill_(GUARD)
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            assert torch.equal(c.y, want)
            c.x.neg_()
            c.run()
            assert not torch.equal(c.y, want)
            c.x.neg_()
