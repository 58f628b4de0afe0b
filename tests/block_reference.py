"""Matrix product with an epilogue and group norm with an activation in 64 bits, and how far a kernel may be from them.

Plain numpy, written from the formulas; no library code.  The bounds count roundings, u = 2^-24 for fp32:

* A sum of K products (exact in fp32 for 16-bit operands) over matrix instructions of depth 32: at most 32 additions inside
  an instruction and K / 32 between instructions, and a few that join partial sums, each off by at most 2 u (the instruction
  may truncate) of the sum of absolute terms A; bias and residual are two more additions.
* The activations' slopes are at most 1.13, and a value v of theirs is computed to within 3e-6 |v| (the polynomial and the
  argument of the exponential of GELU; the others are closer).
* The result is rounded once, by at most half a step: finfo.eps / 2 of it, or half of the smallest subnormal.
"""

import math

import numpy as np
import torch

U = 2.0 ** -24
SLOPE, ACT_REL = 1.13, 3e-6
ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -126}


def activation(v, act):
    if act == "relu":
        return np.where(v < 0, 0.0, v)
    if act == "silu":
        return v / (1.0 + np.exp(-np.clip(v, -700, None)))
    if act == "gelu":
        return v * np.vectorize(lambda t: 0.5 * math.erfc(-t * math.sqrt(0.5)), otypes=[float])(v)
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)))
    return v


def rounded_bound(ref, err, dtype, act):
    """Bound on |got - ref| where the value before the activation is off by at most ``err``."""
    e = err if act in ("none", "relu") else SLOPE * err + ACT_REL * np.abs(ref)
    return e + HALF_STEP[dtype] * (np.abs(ref) + e) + TINY[dtype]


def matmul(x, w, b=None, r=None, act="none"):
    """-> (y, bound on the error of the fp32 value before the activation), float64 arrays."""
    x, w = x.astype(np.float64), w.astype(np.float64)
    v, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    for t in (b, r):
        if t is not None:
            v = v + t.astype(np.float64)
            mag = mag + np.abs(t.astype(np.float64))
    return activation(v, act), 2.0 * U * (32 + x.shape[1] / 32 + 18) * mag


def group_norm(x, gamma, beta, groups, eps, r=None, act="none"):
    """x: (N, H, W, C).  -> (y, bound on the error of the fp32 value before the activation).

    The kernels add a group's values in partial sums of at most 1024 terms joined by trees: any of its sums is off by at
    most (1024 + 40) u of the sum of absolute terms, and typically by a hundredth of that.
    """
    N, H, W, C = x.shape
    cg = C // groups
    s = x.astype(np.float64).reshape(N, H * W, groups, cg)
    mean = s.mean(axis=(1, 3), keepdims=True)
    d = s - mean
    var = (d * d).mean(axis=(1, 3), keepdims=True)
    std = np.sqrt(var + eps)
    g = (np.ones(C) if gamma is None else gamma.astype(np.float64)).reshape(groups, cg)
    b = (np.zeros(C) if beta is None else beta.astype(np.float64)).reshape(groups, cg)
    v = d / std * g + b
    depth = min(H * W * cg, 1024) + 40
    e_mean = depth * U * np.abs(s).mean(axis=(1, 3), keepdims=True)
    # (x - mean') differs by e_mean and its own rounding; their squares' mean by 2 |d| e + e^2 and its sum's roundings
    e_d = e_mean + U * (np.abs(s) + np.abs(mean))
    e_var = (2 * np.abs(d) * e_d + e_d ** 2).mean(axis=(1, 3), keepdims=True) + depth * U * var
    rel_std = e_var / (2 * (var + eps)) + 4 * U
    err = (e_d / std + np.abs(d) / std * (rel_std + 4 * U)) * np.abs(g) + 4 * U * (np.abs(v) + np.abs(b))
    v, err = v.reshape(x.shape), err.reshape(x.shape)
    if r is not None:
        v = v + r.astype(np.float64)
        err = err + 2 * U * (np.abs(v) + np.abs(r))
    return activation(v, act), err


def assert_within(got, ref, bound, what=""):
    got = np.asarray(got, dtype=np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    bad = ~(np.abs(got - ref) <= bound)
    if bad.any():
        i = tuple(int(k[0]) for k in np.nonzero(bad))
        raise AssertionError("%s: %d of %d outside; first at %r: got %r, ref %r, bound %r"
                             % (what, int(bad.sum()), bad.size, i, got[i], ref[i], bound[i]))
