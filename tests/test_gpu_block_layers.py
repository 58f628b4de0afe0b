"""Group norm and per-pixel product layers of models on a gpu-let: what a run refuses before it begins, and what it may use."""

import pytest
import torch

import oracle
from paper_2109_01611_amd import gpulet, lowering, workloads

from gpu_util import MODEL_TOL
from test_abi_host import _desc, _layer
from test_block_layers_host import _reads_its_input_again

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _refused(d, part, x, y, ws, n):
    before = part.kernel_launches()
    with pytest.raises(gpulet.GpuletError) as e:
        gpulet.run_model(d, 1, part, x, y, ws, n)
    assert e.value.status == gpulet.EINVAL and part.kernel_launches() == before
    with pytest.raises(gpulet.GpuletError) as e:
        gpulet.ModelGraph(d, 1, part, x, y, ws, n)
    assert e.value.status == gpulet.EINVAL and part.kernel_launches() == before


@pytest.mark.parametrize("kind", ["norm", "product"])
def test_a_layer_that_refuses_its_tensors_refuses_the_run(kind):
    # a convolution in front: were the layer refused when its turn comes, that one would run already
    C = 16
    w = torch.eye(C, dtype=torch.bfloat16, device=DEV)
    last = dict(op=gpulet.OP_GROUP_NORM, K=4, eps=1e-5) if kind == "norm" else dict(op=gpulet.OP_MATMUL, K=C, w=w.data_ptr())
    d = _desc([_layer(op=gpulet.OP_CONV, in_buf=0, out_buf=2, C=C, K=C, R=1, S=1, stride=1, pad=0, w=w.data_ptr()),
               _layer(in_buf=2, out_buf=1, C=C, **last)], 3, (C, 8, 8))
    n = gpulet.model_workspace_bytes(d, 1)
    x = torch.randn(8, 8, C, device=DEV).bfloat16()
    room = torch.zeros(64 * C + 8, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(n + 4096, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    with gpulet.Partition(0, 100, 0) as part:
        _refused(d, part, x, room.data_ptr() + 1, ws, n)        # not a multiple of an element
        _refused(d, part, x, ws.data_ptr() + 32, ws, n)         # over what the layer reads
        gpulet.run_model(d, 1, part, x, room.data_ptr() + 2, ws, n)
        part.sync()
    y = room[1:1 + 64 * C].view(8, 8, C)
    if kind == "product":
        assert torch.equal(y, x)
    else:
        g = x.double().view(64, 4, 4)
        want = (g - g.mean((0, 2), keepdim=True)) / torch.sqrt(g.var((0, 2), unbiased=False, keepdim=True) + 1e-5)
        assert bool(((y.double().view(64, 4, 4) - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all())


def test_products_use_what_scratch_there_is_and_no_more():
    # 4096 pixels of 1022 channels: both operands are laid out anew where there is room.  Small integers: sums are exact.
    C, K, H = 1022, 1024, 64
    g = torch.Generator().manual_seed(1)
    x = torch.randint(-4, 5, (H * H, C), generator=g).to(DEV).bfloat16()
    w = torch.randint(-4, 5, (K, C), generator=g).to(DEV).bfloat16()
    want = x.float() @ w.float().t()
    d = _desc([_layer(op=gpulet.OP_MATMUL, in_buf=0, out_buf=1, C=C, K=K, out_fp32=1, w=w.data_ptr())], 2, (C, H, H))
    n = gpulet.model_workspace_bytes(d, 1)
    assert n > 0
    y = torch.empty(H * H, K, device=DEV)
    arena = torch.empty(2 * n + y.numel() * 4 + 4096, dtype=torch.uint8, device=DEV)
    with gpulet.Partition(0, 100, 0) as part:
        def run(out, ws, size):
            arena.fill_(0xFF)
            y.fill_(-1.0)
            torch.cuda.synchronize()
            gpulet.run_model(d, 1, part, x, out, ws, size)
            part.sync()
            launched = part.kernel_launches()
            return launched
        before = part.kernel_launches()
        for size, launches in ((n, 2), (2 * n, 2), (n // 2 // 256 * 256, 1), (0, 1)):
            now = run(y, arena if size else None, size)
            assert torch.equal(y, want) and now - before == launches, size
            assert bool((arena[n:] == 0xFF).all())          # nothing behind what the model asks for
            before = now
        # the output inside of the scratch, at its start and further back
        for at, launches in ((0, 1), (512, 1), (n, 2)):
            out = arena[at:at + y.numel() * 4].view(torch.float32).view(H * H, K)
            now = run(out, arena, arena.numel() // 256 * 256)
            assert torch.equal(out, want) and now - before == launches, at
            before = now
        graph_ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
        graph = gpulet.ModelGraph(d, 1, part, x, y, graph_ws, n)
        for _ in range(3):
            y.fill_(-1.0)
            torch.cuda.synchronize()
            graph.launch()
            part.sync()
            assert torch.equal(y, want)
        graph.destroy()


def test_a_model_that_reads_its_input_again():
    model = _reads_its_input_again()
    params, x = workloads.parameters(model, 3), workloads.batch_input(model, 3, 3)
    dm = lowering.DeviceModel(model, params, DEV)
    with gpulet.Partition(0, 100, 0) as part:
        y, _ = dm.run(part, dm.input_to_device(x))
    want = oracle.run_model(model, params, x)
    assert max(oracle.rel_err(lowering.nhwc_to_nchw(y), want)) <= MODEL_TOL
