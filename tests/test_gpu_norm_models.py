"""The residual network of group norm, convolution and per-pixel product layers on a gpu-let: each layer on its actual input,
the whole against the oracle, eager against graph replays, batches and gpu-lets that change nothing, launches counted."""

import numpy as np
import pytest
import torch

import block_reference as ref
import oracle
from paper_2109_01611_amd import gpulet, lowering, workloads

from gpu_util import DEV, MODEL_TOL, assert_close, conv_mag

pytestmark = pytest.mark.gpu
NETS = [workloads.norm_residual((16, 24), blocks=2, in_hw=17, n_class=5), workloads.norm_residual((64, 128, 256), in_hw=96),
        workloads.norm_residual((320,), groups=32, in_hw=128)]


def _run(model, batch, seed=0, pct=100, **kw):
    params, x = workloads.parameters(model, seed), workloads.batch_input(model, batch, seed)
    dm = lowering.DeviceModel(model, params, DEV, **kw)
    with gpulet.Partition(0, pct, 0) as part:
        y, _ = dm.run(part, dm.input_to_device(x))
        n = part.kernel_launches()
    return dm, params, x, y, n


@pytest.mark.parametrize("model", NETS, ids=lambda m: m.name)
def test_whole_network(model):
    for batch in (1, 3):
        dm, params, x, y, launches = _run(model, batch)
        got = y.cpu().numpy().astype(np.float64)
        assert got.shape == (batch, 1, 1, got.shape[3]) and y.dtype == torch.float32
        want = oracle.run_model(model, params, x)
        whole, per = oracle.rel_err(got.transpose(0, 3, 1, 2), want)
        assert max(whole, per) <= MODEL_TOL, (whole, per)
        assert launches >= len(dm.layers) - 3       # convolutions may share launches, large norms take two


@pytest.mark.parametrize("model", NETS[:2], ids=lambda m: m.name)
def test_every_layer_on_its_actual_input(model):
    batch = 2
    dm, params, x, y, _ = _run(model, batch, seed=1, reuse=False, merge_siblings=False)
    t = {"x": x.astype(np.float64)}
    for nd in model.nodes:
        a, src = nd.attr, t[nd.src]
        if nd.dst == model.out:
            got = y.cpu().numpy().astype(np.float64).transpose(0, 3, 1, 2)
        else:
            got = dm.read_tensor(nd.dst, batch).float().cpu().numpy().astype(np.float64).transpose(0, 3, 1, 2)
        res = t[a["residual"]] if a.get("residual") else None
        nhwc = lambda v: v.transpose(0, 2, 3, 1)
        if nd.op == "conv":
            w, b = params[nd.name]
            assert_close(got, oracle.conv2d(src, w, b, a["stride"], a["pad"], a["relu"], res),
                         conv_mag(src, w, b, a["stride"], a["pad"], res), what=nd.name)
        elif nd.op in ("groupnorm", "matmul"):
            w, b = params[nd.name]
            dt = torch.float32 if nd.dst == model.out else torch.bfloat16
            if nd.op == "groupnorm":
                want, err = ref.group_norm(nhwc(src), np.asarray(w), np.asarray(b), a["groups"], a["eps"],
                                           None if res is None else nhwc(res), a["act"])
            else:
                rows = nhwc(src).reshape(-1, a["C"])
                want, err = ref.matmul(rows, np.asarray(w), np.asarray(b), None if res is None else nhwc(res).reshape(-1, a["K"]), a["act"])
                want, err = (v.reshape(nhwc(got).shape) for v in (want, err))
            ref.assert_within(nhwc(got), want, ref.rounded_bound(want, err, dt, a["act"]), nd.name)
        t[nd.dst] = got


@pytest.mark.parametrize("model", NETS, ids=lambda m: m.name)
def test_graph_replays_match_eager(model):
    batch = 2
    params, x = workloads.parameters(model, 2), workloads.batch_input(model, batch, 2)
    dm = lowering.DeviceModel(model, params, DEV)
    other = lowering.DeviceModel(NETS[0], workloads.parameters(NETS[0], 3), DEV)
    xo = other.input_to_device(workloads.batch_input(NETS[0], 4, 3))
    with gpulet.Partition(0, 50, 0) as p:
        xd = dm.input_to_device(x)
        want = dm.run(p, xd)[0].clone()
        n = gpulet.model_workspace_bytes(dm.desc, batch)
        graphs, outs, keep = [], [], []
        for _ in range(2):               # a workspace of its own for each graph
            ws = torch.full((max(n, 256),), 0xFF, dtype=torch.uint8, device=DEV)
            y = dm.alloc_output(batch)
            torch.cuda.synchronize()
            graphs.append(gpulet.ModelGraph(dm.desc, batch, p, xd, y, ws, n))
            outs.append(y)
            keep.append(ws)
        for i in range(4):
            for g, y in zip(graphs, outs):
                y.fill_(-1.0)
                torch.cuda.synchronize()
                g.launch()
            p.sync()
            assert torch.equal(outs[0], want) and torch.equal(outs[1], want), i
            other.run(p, xo)
            torch.cuda.synchronize()
        for g in graphs:
            g.destroy()


def test_gpu_let_sizes_and_profile():
    model = NETS[1]
    params, x = workloads.parameters(model, 4), workloads.batch_input(model, 2, 4)
    dm = lowering.DeviceModel(model, params, DEV)
    want = oracle.run_model(model, params, x)
    for pct in (20, 60):
        with gpulet.Partition(0, pct, 0) as p:
            xd = dm.input_to_device(x)
            y, _ = dm.run(p, xd)
            assert oracle.rel_err(y.cpu().numpy().astype(np.float64).transpose(0, 3, 1, 2), want)[1] <= MODEL_TOL
            ws, n = dm.workspace(2)
            lat, total = gpulet.profile_model(dm.desc, 2, p, xd, y, ws, n, 2, 5)
            assert len(lat) == 5 and min(lat) > 0


def test_scratch_may_not_overlap_input_or_output():
    C = 16
    L = gpulet.Layer()
    L.op, L.in_buf, L.out_buf, L.res_buf, L.C, L.K, L.eps = gpulet.OP_GROUP_NORM, 0, 1, -1, C, 1, 1e-5
    d = gpulet.ModelDesc()
    d.n_layers, d.n_bufs, d.in_C, d.in_H, d.in_W, d.in_buf, d.out_buf = 1, 2, C, 256, 256, 0, 1
    d.layers = (gpulet.Layer * 1)(L)
    n = gpulet.model_workspace_bytes(d, 1)
    x = torch.randn(256, 256, C, device=DEV).bfloat16()
    y = torch.empty_like(x)
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)
    with gpulet.Partition(0, 100, 0) as p:
        for bad in ((x, y, x), (x, y, y)):
            with pytest.raises(gpulet.GpuletError) as e:
                gpulet.run_model(d, 1, p, bad[0], bad[1], bad[2].data_ptr(), n)
            assert e.value.status == gpulet.EINVAL
        with pytest.raises(gpulet.GpuletError) as e:
            gpulet.run_model(d, 1, p, x, y, ws, n - 1)
        assert e.value.status == gpulet.ENOMEM
        # a misaligned input takes narrower loads and no more scratch than was asked for
        flat = torch.empty(x.numel() + 1, dtype=torch.bfloat16, device=DEV)
        flat[1:].copy_(x.view(-1))
        torch.cuda.synchronize()
        gpulet.run_model(d, 1, p, flat.data_ptr() + 2, y, ws, n)
        p.sync()
    want, err = ref.group_norm(x.double().cpu().numpy()[None], None, None, 1, 1e-5)
    ref.assert_within(y.double().cpu().numpy()[None], want, ref.rounded_bound(want, err, torch.bfloat16, "none"))
