"""How far a group norm kernel may be from the definition when what it sums are differences from a value near the mean.

``block_reference.group_norm`` lets the mean be off by the roundings of a sum of the values themselves, which for a mean of
1000 standard deviations is several percent of one.  The kernels' sums are of differences, so that a mean's error is

* the roundings of a sum of differences, at most 1024 + 40 of u = 2^-24 each of the mean absolute difference, and
* the roundings of the mean itself, u |mean| each: one per batch of a thread (32 at most), per value joined by a lane
  (16 in a workgroup, the same for the chunks of an image up to 1024 of them) and per level of the two trees of 64 lanes.

A partial mean that is off by e changes the squared differences by 2 |d| e + e^2, as in block_reference.
"""

import numpy as np

import block_reference as ref

U = ref.U
MEAN_ROUNDINGS = 32 + 2 * (16 + 6)


def group_norm(x, gamma, beta, groups, eps, r=None, act="none"):
    """x: (N, H, W, C).  -> (y, bound on the error of the fp32 value before the activation)."""
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
    e_mean = depth * U * np.abs(d).mean(axis=(1, 3), keepdims=True) + MEAN_ROUNDINGS * U * np.abs(mean)
    e_d = e_mean + U * np.abs(d)
    e_var = (2 * np.abs(d) * e_d + e_d ** 2).mean(axis=(1, 3), keepdims=True) + depth * U * var
    rel_std = e_var / (2 * (var + eps)) + 4 * U
    err = (e_d / std + np.abs(d) / std * (rel_std + 4 * U)) * np.abs(g) + 4 * U * (np.abs(v) + np.abs(b))
    v, err = v.reshape(x.shape), err.reshape(x.shape)
    if r is not None:
        v = v + r.astype(np.float64)
        err = err + 2 * U * (np.abs(v) + np.abs(r))
    return ref.activation(v, act), err
