"""Group norm and per-pixel product layers of models without a GPU: what they share, what a run plans and what it refuses."""

import time

import pytest

from paper_2109_01611_amd import gpulet, lowering, workloads

from test_abi_host import _desc, _layer
from test_model_lanes_host import _happens_before

W = 1 << 40   # stand-in address, never followed


def _conv(i, o):
    return _layer(op=gpulet.OP_CONV, in_buf=i, out_buf=o, C=16, K=16, R=1, S=1, stride=1, pad=0, w=W)


def _norm(i, o, **kw):
    return _layer(op=gpulet.OP_GROUP_NORM, in_buf=i, out_buf=o, C=16, K=1, eps=1e-5, **kw)


def _product(i, o, C=16, K=16, **kw):
    return _layer(op=gpulet.OP_MATMUL, in_buf=i, out_buf=o, C=C, K=K, w=W, **kw)


@pytest.mark.parametrize("kinds", ["nn", "nm", "mn", "mm", "ncn", "nnmm", "mnmn"])
def test_layers_that_share_scratch_are_ordered_on_two_lanes(kinds):
    # branches from one tensor, each layer on a buffer of its own: without the scratch nothing would order them
    make = dict(n=_norm, m=_product, c=_conv)
    layers = [_conv(0, 2)] + [make[k](2, 3 + i) for i, k in enumerate(kinds)]
    layers += [_product(3 + i, 3 + len(kinds) + i if i + 1 < len(kinds) else 1) for i in range(len(kinds))]
    d = _desc(layers, 3 + 2 * len(kinds), (16, 256, 256))
    assert gpulet.model_workspace_bytes(d, 1) > 0
    lane, waits = gpulet.model_schedule(d, 1, lanes=2)
    reach = _happens_before(len(layers), lane, waits)
    users = [i for i, L in enumerate(layers) if L.op in (gpulet.OP_GROUP_NORM, gpulet.OP_MATMUL)]
    for a, i in enumerate(users):
        for j in users[a + 1:]:
            assert i in reach[j], (i, j, lane, waits)
    if "c" in kinds:
        assert set(lane) == {0, 1}       # a convolution beside them still goes where there is room
    assert gpulet.model_schedule(d, 1, lanes=1) == ([0] * len(layers), [])


def _seconds(f, n=30):
    best = 1.0
    for _ in range(n):
        t = time.perf_counter()
        f()
        best = min(best, time.perf_counter() - t)
    return best


def test_a_run_does_not_look_through_all_numbers_of_cus():
    # What a run plans (also for the shape of a buffer) against what the size of the workspace takes, which looks for every
    # product through 32 numbers of CUs: before runs left that out, the two took the same time.
    n = 24
    layers = [_product(0 if i == 0 else 1 + i, 2 + i if i + 1 < n else 1, 256, 256) for i in range(n)]
    d = _desc(layers, n + 1, (256, 24, 24))
    run = _seconds(lambda: gpulet.model_buffer_info(d, 2, 1))
    size = _seconds(lambda: gpulet.model_workspace_bytes(d, 2))
    assert run < 0.5 * size, (run, size)


def test_workspace_still_holds_what_products_are_fastest_with():
    # 4096 x 4096 pixels' products of a depth that is no multiple of 8: copies of both operands
    mm = gpulet.matmul_desc(1 << 41, 1 << 42, None, 1 << 43, 64 * 64, 4096, 1022)
    need = gpulet.matmul_workspace_bytes(mm)
    assert need > 0
    d = _desc([_product(0, 1, 1022, 4096)], 2, (1022, 64, 64))
    assert gpulet.model_workspace_bytes(d, 1) == (need + 255) // 256 * 256


def _reads_its_input_again():
    n = workloads
    nodes = [n._conv("a", "x", "a", 3, 16, 3, 1, 1, False), n._groupnorm("g", "a", "b", 16, 4, "silu"),
             n._matmul("m", "b", "c", 16, 3, residual="x"), n._groupnorm("h", "c", "d", 3, 1, residual="x"),
             n._conv("e", "x", "e", 3, 8, 3, 1, 1, False), n._conv("f", "d", "y", 3, 8, 3, 1, 1, True, residual="e")]
    return n.Model("input_again", (3, 10, 10), "normal", nodes, "y")


def test_the_models_input_as_a_residual_is_not_padded():
    # convolutions of the input get zero channels, which a residual of three channels has not
    model = _reads_its_input_again()
    dm = lowering.DeviceModel(model, workloads.parameters(model, 0), "cpu")
    assert dm.in_pad == 0 and gpulet.model_workspace_bytes(dm.desc, 2) > 0
    plain = model._replace(nodes=[nd._replace(attr=dict(nd.attr, residual=None)) if nd.attr.get("residual") == "x" else nd
                                  for nd in model.nodes])
    assert lowering.DeviceModel(plain, workloads.parameters(plain, 0), "cpu").in_pad == 1
