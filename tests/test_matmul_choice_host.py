"""Which form a matrix product runs in, asked of the library on the CPU, and that the sizes of the GPU tests reach them all."""

import os
import shutil
import subprocess

import pytest

import test_gpu_matmul
from paper_2109_01611_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
FORMS = ("ring11", "ring11w", "ring12", "ring22", "ring42", "ring44", "tile64", "tile128x64", "tile128", "big", "direct", "direct22",
         "staged")
PLENTY = 1 << 40


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    hipcc = shutil.which("hipcc")
    if not hipcc:
        pytest.skip("no hipcc")
    exe = str(tmp_path_factory.mktemp("forms") / "record")
    lib = os.path.dirname(build.LIB)
    subprocess.run([hipcc, "-O1", "-std=c++17", "-w", "-x", "hip", "--cuda-host-only", "-I", os.path.join(build.ROOT, "include"),
                    "-I", build.CSRC, os.path.join(HERE, "native", "record_matmul_forms.cpp"), "-x", "none", "-o", exe,
                    "-L", lib, "-lgpulet", "-Wl,-rpath," + lib], check=True, timeout=300)

    def ask(cases):
        """[(M, N, K, more)] with more: n_cu, ldx, shift, ws -> [(form, split, rows laid out anew)]"""
        text = ""
        for M, N, K, more in cases:
            m = dict(n_cu=256, ldx=0, shift=0, ws=0)
            m.update(more)
            text += "%d %d %d %d %d %d %d\n" % (m["n_cu"], M, N, K, m["ldx"], m["shift"], m["ws"])
        out = subprocess.run([exe], input=text, capture_output=True, text=True, timeout=60, check=True).stdout.split("\n")[:-1]
        assert len(out) == len(cases)
        return [(FORMS[int(f)], int(k), bool(int(c))) for f, k, c in (line.split() for line in out)]
    return ask


def test_gpu_sizes_reach_every_form(choose):
    cases = [s + (dict(ws=PLENTY),) for s in test_gpu_matmul.SIZES]
    got = choose(cases + [s + ({},) for s in test_gpu_matmul.SIZES] + [s[:3] + (dict(shift=1, ws=PLENTY),) for s in cases])
    assert {f for f, _, _ in got} == set(FORMS)
    assert {f for f, k, _ in got if k > 1} == {"tile64"} and {f for f, _, c in got if c} >= {"ring42", "tile64", "big"}


def test_unaligned_rows_never_use_transfers(choose):
    sizes = [(1, 64, 64), (40, 640, 512), (300, 300, 4096), (4096, 4096, 4096)]
    for more in (dict(shift=1), dict(shift=2), dict(shift=4), dict(ldx=4097), dict(ldx=4100)):
        for f, k, c in choose([s + (more,) for s in sizes]):
            assert f in ("direct", "direct22", "staged") and k == 1 and not c
        # ... unless there is room to lay them out anew, and then only large ones
        got = choose([s + (dict(more, ws=PLENTY),) for s in sizes])
        assert not got[0][2] and got[-1] == ("big", 1, True)
    for f, _, c in choose([(M, N, K + 4, {}) for M, N, K in sizes]):     # a depth that is not a multiple of 8
        assert f in ("direct", "direct22", "staged") and not c
    for f, _, c in choose([s + (dict(ldx=8192, ws=PLENTY),) for s in sizes]):
        assert f not in ("direct", "direct22", "staged") and not c
    # exactly enough room, and a byte less
    M, N, K = 4096, 4096, 4090
    both, x_only = 2 * (M + N) * 4096, 2 * M * 4096
    assert choose([(M, N, K, dict(ws=both))])[0][2] and not choose([(M, N, K, dict(ws=both - 1))])[0][2]
    assert choose([(M, N, 4096, dict(ldx=4097, ws=x_only))])[0][2] and not choose([(M, N, 4096, dict(ldx=4097, ws=x_only - 1))])[0][2]


def test_shared_depth_only_with_room_for_the_sums(choose):
    M, N, K = 5470, 88, 8192
    plane = 4 * M * N
    assert choose([(M, N, K, {})])[0][1] == 1
    splits = [choose([(M, N, K, dict(ws=n))])[0][1] for n in (2 * plane - 1, 2 * plane, 4 * plane, PLENTY)]
    assert splits[0] == 1 and all(k * plane <= max(n, plane) for k, n in zip(splits, (0, 2 * plane, 4 * plane, PLENTY)))
    assert splits[-1] > 1


def test_few_rows_and_very_wide_or_tall(choose):
    for M in (1, 2, 16, 17, 64):
        for N in (8, 1000, 131072, 1 << 20):
            f, _, _ = choose([(M, N, 1024, {})])[0]
            assert f.startswith("ring") or f.startswith("tile"), (M, N, f)
    # more workgroups of 16 x 16 than a grid can hold
    assert choose([(1 << 24, 32, 64, {})])[0][0] in ("tile64", "tile128x64", "tile128", "big")
    assert choose([(8192, 8192, 8192, {})])[0][0] == "big"
