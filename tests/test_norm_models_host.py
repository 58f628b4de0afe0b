"""Group norm and per-pixel product layers of models without a GPU: the oracle's definitions against torch in float64, what a
description may say, the workspace behind the buffers, and the lowering of the residual network."""

import numpy as np
import pytest
import torch

import oracle
from paper_2109_01611_amd import gpulet, lowering, profiler, workloads

from test_abi_host import _desc, _layer

W = 4096
NET = workloads.norm_residual((16, 24), blocks=2, in_hw=16, n_class=5)


def test_oracle_group_norm_and_product_match_torch_in_float64():
    rng = np.random.default_rng(0)
    x, r = rng.standard_normal((2, 12, 5, 7)) * 3 + 1, rng.standard_normal((2, 12, 5, 7))
    g, b = rng.standard_normal(12), rng.standard_normal(12)
    t = lambda a: torch.from_numpy(a)
    F = torch.nn.functional
    acts = {"none": lambda v: v, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}
    for act, f in acts.items():
        for groups in (1, 3, 12):
            want = f(F.group_norm(t(x), groups, t(g), t(b), 1e-3) + t(r)).numpy()
            np.testing.assert_allclose(oracle.group_norm(x, g, b, groups, 1e-3, act, r), want, rtol=1e-10, atol=1e-12)
        w, c = rng.standard_normal((9, 12)), rng.standard_normal(9)
        want = f(F.conv2d(t(x), t(w)[:, :, None, None], t(c))).numpy()
        np.testing.assert_allclose(oracle.pixel_matmul(x, w, c, act), want, rtol=1e-10, atol=1e-12)


def test_network_table_is_consistent():
    params = workloads.parameters(NET, 0)
    assert oracle.model_params(NET) == sum(np.asarray(w).size + np.asarray(b).size for w, b in params.values())
    assert profiler.model_flops(NET) == oracle.model_flops(NET)
    y = oracle.run_model(NET, params, workloads.batch_input(NET, 2, 0))
    assert y.shape == (2, 5, 1, 1) and np.isfinite(y).all()


def test_lowered_network_is_accepted_and_buffers_are_reused():
    dm = lowering.DeviceModel(NET, workloads.parameters(NET, 0), "cpu")
    plain = lowering.DeviceModel(NET, workloads.parameters(NET, 0), "cpu", reuse=False)
    ops = [L.op for L in dm.layers]
    assert ops.count(gpulet.OP_GROUP_NORM) == 13 and ops.count(gpulet.OP_MATMUL) == 9
    assert dm.out_fp32 and dm.layers[len(ops) - 1].out_fp32 == 1
    for batch in (1, 7):
        assert 0 < gpulet.model_workspace_bytes(dm.desc, batch) < gpulet.model_workspace_bytes(plain.desc, batch)
        assert gpulet.model_buffer_info(dm.desc, batch, 1)[:4] == (5, 1, 1, 4)
    # a residual is never in a buffer that something between its writer and its reader overwrites
    value = {0: "x"}
    for L, nd in zip(dm.layers, [n for n in NET.nodes if n.op != "concat"]):
        assert value[L.in_buf] == nd.src
        if nd.attr.get("residual"):
            assert value[L.res_buf] == nd.attr["residual"]
        value[L.out_buf] = nd.dst


def test_descriptions():
    norm = dict(op=gpulet.OP_GROUP_NORM, in_buf=0, out_buf=1, C=16, K=4, relu=gpulet.ACT_SILU, eps=1e-5)
    mm = dict(op=gpulet.OP_MATMUL, in_buf=0, out_buf=1, C=16, K=24, relu=gpulet.ACT_GELU, w=W)
    conv = _layer(op=gpulet.OP_CONV, in_buf=0, out_buf=2, C=16, K=16, R=1, S=1, stride=1, pad=0, w=W)

    def ask(layers, n_bufs=2, shape=(16, 6, 6), batch=3):
        return gpulet.model_workspace_bytes(_desc(layers, n_bufs, shape), batch)
    assert ask([_layer(**norm)]) == 0
    assert ask([_layer(**mm)]) == 0
    assert gpulet.model_buffer_info(_desc([_layer(**mm)], 2, (16, 6, 6)), 3, 1)[:4] == (24, 6, 6, 2)
    assert gpulet.model_buffer_info(_desc([_layer(out_fp32=1, **mm)], 2, (16, 6, 6)), 3, 1)[:4] == (24, 6, 6, 4)
    buffers = 3 * 16 * 6 * 6 * 2
    assert ask([conv, _layer(res_buf=2, **norm)], 3) == (buffers + 255) // 256 * 256
    # a large map needs scratch behind the buffers, the largest of its layers'
    big = dict(norm, K=1)
    scratch = ask([_layer(**big)], shape=(16, 256, 256))
    assert scratch > 0 and scratch % 256 == 0
    d = gpulet.group_norm_desc(1 << 40, None, None, 1 << 41, 3, 16, 256, 256, 1)
    assert gpulet.group_norm_workspace_bytes(d) <= scratch
    bad = [dict(norm, C=8), dict(norm, K=3), dict(norm, K=0), dict(norm, eps=-1.0), dict(norm, relu=5), dict(norm, res_buf=2),
           dict(norm, in_buf=1), dict(norm, w=W + 2), dict(mm, C=8), dict(mm, K=0), dict(mm, w=None), dict(mm, relu=-1), dict(mm, res_buf=2),
           dict(mm, w=W + 1), dict(mm, group_next=1)]
    for kw in bad:
        with pytest.raises(gpulet.GpuletError) as e:
            ask([_layer(**kw)], 3)
        assert e.value.status == gpulet.EINVAL, kw
    for kw in (dict(mm, res_buf=2), dict(mm, K=16, out_fp32=1, res_buf=2)):     # 16 channels for 24; bf16 for fp32
        with pytest.raises(gpulet.GpuletError) as e:
            ask([conv, _layer(**kw)], 3)
        assert e.value.status == gpulet.EINVAL, kw
    # an fp32 tensor is an output, nothing reads it
    with pytest.raises(gpulet.GpuletError):
        ask([_layer(**dict(mm, out_buf=2, K=16, out_fp32=1)), _layer(**dict(norm, in_buf=2))], 3)


def test_concat_slices_are_not_read_as_residuals():
    n = workloads
    nodes = [n._conv("a", "x", "a", 16, 8, 1), n._conv("b", "x", "b", 16, 8, 1), n._concat("c", ["a", "b"], "c"),
             n._conv("d", "c", "d", 16, 8, 1), n._groupnorm("g", "d", "y", 8, 2, residual="a")]
    m = n.Model("bad", (16, 4, 4), "normal", nodes, "y")
    with pytest.raises(ValueError):
        lowering.DeviceModel(m, n.parameters(m, 0), "cpu")
