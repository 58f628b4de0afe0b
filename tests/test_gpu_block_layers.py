"""Group norm and per-pixel product layers of models on a gpu-let: what a run refuses before it begins, and what it may use."""

import pytest
import torch

from paper_2109_01611_amd import gpulet

from test_abi_host import _desc, _layer

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
