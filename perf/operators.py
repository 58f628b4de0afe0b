"""The matrix product with an epilogue and group norm with an activation, as measurable cases.

Both are layers of served networks that a 1x1 convolution or a folded batch norm cannot stand for:

  matmul      y[m, n] = act(sum_k x[m, k] w[n, k] + b[n] + r[m, n])
  group_norm  y = act((x - mean) / sqrt(var + eps) * gamma[c] + beta[c] + r), mean and var per image and group of
              channels, x in NHWC order

``run`` computes them in elementary torch operations, or, where ``own`` is set, with the library's calls on the current
stream, the way a serving executor makes them: weights, workspace, output and descriptor are set up once.
"""

import math

import torch

own = False
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
EPS = 1e-5


def _mm(name, M, N, K, dtype="bf16", out="bf16", act="none", bias=True, res=False, ldx=0):
    """``ldx``: elements between rows of x where x is a slice of wider rows (0: dense)."""
    return dict(name=name, op="matmul", M=M, N=N, K=K, dtype=dtype, out=out, act=act, bias=bias, res=res, ldx=ldx)


def _gn(name, N, H, W, C, G, dtype="bf16", act="silu", res=False, ldx=0):
    """``ldx``: channels per stored pixel where x is a channel slice of wider pixels (0: dense)."""
    return dict(name=name, op="group_norm", N=N, H=H, W=W, C=C, G=G, dtype=dtype, act=act, res=res, ldx=ldx)


def listed():
    return [
        # one request through a hidden classifier layer (VGG's fc7): the weights are read once, latency counts
        _mm("mm_one_row", 1, 4096, 4096, act="relu"),
        # a batch of single rows back to the narrow width, into the residual stream
        _mm("mm_24_rows", 24, 1024, 4096, dtype="f16", out="f16", res=True),
        # one image's pixels, nothing a multiple of anything, logits kept in 32 bits
        _mm("mm_odd", 787, 333, 1001, out="f32", act="gelu"),
        # the wide half of a block on the pixels of a 14x14 map at batch 11, read out of wider rows
        _mm("mm_up_slice", 2156, 2560, 640, act="silu", ldx=1280),
        # and its narrow half on a full batch, with the shortcut
        _mm("mm_down", 6272, 1024, 4096, res=True),
        # a large map at a full batch: nothing but matrix instructions
        _mm("mm_large", 8192, 4096, 4096, act="gelu_tanh"),
        # the bottom of a network for one request: a few microseconds, all of it latency
        _gn("gn_one_8x8", 1, 8, 8, 1280, 32),
        # one image in the middle of the network, 10 channels a group, half of a concatenated tensor
        _gn("gn_one_64x64_slice", 1, 64, 64, 320, 32, ldx=640),
        # an ordinary batch with the shortcut in front of the ReLU (a ResNet stage)
        _gn("gn_resnet_14x14", 32, 14, 14, 1024, 32, act="relu", res=True),
        # nothing a multiple of anything, 32 bits
        _gn("gn_odd", 5, 37, 29, 246, 6, dtype="f32", act="gelu"),
        # a batch at 64 x 64
        _gn("gn_b16_64x64", 16, 64, 64, 320, 32, dtype="f16"),
        # full-resolution maps: memory traffic only
        _gn("gn_b8_256x256", 8, 256, 256, 128, 32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of features: mostly multiples of 8, as networks have them, some odd ones."""
    n = _log_int(rng, lo, hi)
    return n if rng.random() < 0.2 else max(8, (n + 4) // 8 * 8)


def draw(rng):
    limit = max(_cost(c) for c in listed())
    while True:
        if rng.random() < 0.5:
            dtype = rng.choice(("bf16", "bf16", "f16"))
            K = _width(rng, 64, 8192)
            c = _mm(None, _log_int(rng, 1, 16384), _width(rng, 32, 8192), K, dtype=dtype,
                    out=rng.choice((dtype, dtype, "f32")), act=rng.choice(ACTS), bias=rng.random() < 0.8,
                    res=rng.random() < 0.4, ldx=2 * K if rng.random() < 0.2 else 0)
        else:
            G = rng.choice((1, 8, 16, 32, 32, 32))
            C = G * _log_int(rng, 2, max(2, 1536 // G))
            c = _gn(None, _log_int(rng, 1, 32), _log_int(rng, 4, 256), _log_int(rng, 4, 256), C, G,
                    dtype=rng.choice(("bf16", "bf16", "f16", "f32")), act=rng.choice(ACTS), res=rng.random() < 0.3,
                    ldx=2 * C if rng.random() < 0.2 else 0)
        del c["name"]
        if _cost(c) <= limit:
            return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / 1e15


def work(case):
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": 2 * (M * K + N * K) + 4 * N * case["bias"] + out * M * N * (2 if case["res"] else 1),
                "flops": 2 * M * N * K}
    n = case["N"] * case["H"] * case["W"] * case["C"]
    size = 4 if case["dtype"] == "f32" else 2
    return {"bytes": size * n * (3 if case["res"] else 2) + 8 * case["C"], "flops": 10 * n}


def _inputs(case, seed):
    """The operands on the GPU; x is a view where it is part of wider rows."""
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEVICE)
    t = TYPES[case["dtype"]]
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        x = normal(M, case["ldx"] or K).to(t)[:, :K]
        w = (normal(N, K) / math.sqrt(K)).to(t)
        b = 0.1 * normal(N) if case["bias"] else None
        r = normal(M, N).to(TYPES[case["out"]]) if case["res"] else None
        return x, w, b, r
    N, H, W, C = case["N"], case["H"], case["W"], case["C"]
    L = case["ldx"] or C
    # channels have means and scales of their own, as the outputs of a convolution with a bias have
    x = normal(N, H, W, L).mul_(0.5 + torch.rand(L, generator=g, device=DEVICE)).add_(normal(L)).to(t)[..., :C]
    gamma, beta = 1.0 + 0.2 * normal(C), 0.2 * normal(C)
    r = normal(N, H, W, C).to(t) if case["res"] else None
    return x, gamma, beta, r


def prepare(case, seed):
    a, b, c, r = _inputs(case, seed)
    state = dict(case=case, args=(a, b, c, r))
    if not own:
        return state
    from paper_2109_01611_amd import gpulet
    types = {"bf16": gpulet.BF16, "f16": gpulet.F16, "f32": gpulet.F32}
    act = {"none": gpulet.ACT_NONE, "relu": gpulet.ACT_RELU, "silu": gpulet.ACT_SILU, "gelu": gpulet.ACT_GELU,
           "gelu_tanh": gpulet.ACT_GELU_TANH}[case["act"]]
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        y = torch.empty((M, N), dtype=TYPES[case["out"]], device=DEVICE)
        desc = gpulet.matmul_desc(a.data_ptr(), b, c, y, M, N, K, act=act, residual=r, ldx=case["ldx"],
                                  dtype=types[case["dtype"]], out_dtype=types[case["out"]])
        call, size = gpulet.matmul, gpulet.matmul_workspace_bytes(desc)
    else:
        y = torch.empty((case["N"], case["H"], case["W"], case["C"]), dtype=a.dtype, device=DEVICE)
        desc = gpulet.group_norm_desc(a.data_ptr(), b, c, y, case["N"], case["C"], case["H"], case["W"], case["G"],
                                      eps=EPS, act=act, residual=r, x_ch_stride=case["ldx"],
                                      dtype=types[case["dtype"]])
        call, size = gpulet.group_norm, gpulet.group_norm_workspace_bytes(desc)
    workspace = torch.empty(size, dtype=torch.uint8, device=DEVICE) if size else None
    state.update(call=call, desc=desc, y=y, workspace=workspace, workspace_bytes=size)
    return state


def run(state):
    if own:
        state["call"](state["desc"], state["workspace"], state["workspace_bytes"],
                      torch.cuda.current_stream().cuda_stream)
        return state["y"]
    case = state["case"]
    if case["op"] == "matmul":
        x, w, b, r = state["args"]
        v = torch.matmul(x.float(), w.float().t())
        if b is not None:
            v = v + b
        out = TYPES[case["out"]]
    else:
        x, gamma, beta, r = state["args"]
        N, H, W, C, G = case["N"], case["H"], case["W"], case["C"], case["G"]
        v = x.float().reshape(N, H * W, G, C // G)
        v = v - v.mean(dim=(1, 3), keepdim=True)
        v = v * torch.rsqrt((v * v).mean(dim=(1, 3), keepdim=True) + EPS)
        v = v.reshape(N, H, W, C) * gamma + beta
        out = x.dtype
    if r is not None:
        v = v + r.float()
    return _act(v, case["act"]).to(out)


def _act(v, act):
    if act == "relu":
        return torch.clamp_min(v, 0.0)
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def exact(case, seed):
    a, b, c, r = _inputs(case, seed)
    if case["op"] == "matmul":
        s = a.double() @ b.double().t().contiguous()
        if c is not None:
            s += c.double()
    else:
        N, H, W, C, G = case["N"], case["H"], case["W"], case["C"], case["G"]
        s = a.double().view(N, H * W, C) if a.is_contiguous() else a.double().reshape(N, H * W, C)
        per = H * W * (C // G)
        mean = (s.sum(dim=1).view(N, G, C // G).sum(dim=2) / per).repeat_interleave(C // G, dim=1)
        s = s - mean[:, None, :]
        var = ((s * s).sum(dim=1).view(N, G, C // G).sum(dim=2) / per).repeat_interleave(C // G, dim=1)
        s = s / torch.sqrt(var + EPS)[:, None, :] * b.double() + c.double()
        s = s.view(N, H, W, C)
    if r is not None:
        s = s + r.double()
    if case["act"] == "relu":
        return torch.where(s > 0, s, torch.zeros_like(s))
    if case["act"] == "silu":
        return s * torch.sigmoid(s)
    if case["act"] == "gelu":
        return s * 0.5 * torch.special.erfc(-s / math.sqrt(2.0))
    if case["act"] == "gelu_tanh":
        return s * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (s + 0.044715 * s ** 3))
    return s
