"""The kernels that the shapes of the GPU tests reach (mx_shapes.py), read from the library's own rules, which a host
program built with g++ and the sanitizers prints.  No GPU is involved."""
import os
import shutil
import subprocess
from pathlib import Path

import pytest

from mx_shapes import GATED, LINEAR

ROOT = Path(__file__).resolve().parents[1]
ROCM_INCLUDE = Path(os.environ.get("ROCM_PATH", "/opt/rocm")) / "include"


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None or not (ROCM_INCLUDE / "hip" / "hip_runtime.h").exists():
        pytest.skip("g++ or the HIP headers are not available")
    exe = tmp_path_factory.mktemp("mx_plan") / "mx_plan_check"
    subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", f"-I{ROCM_INCLUDE}", f"-I{ROOT / 'include'}",
                    f"-I{ROOT / 'paper_2607_14618_amd' / 'csrc'}", str(ROOT / "tests" / "host" / "mx_plan_check.cpp"),
                    "-o", str(exe)], check=True, capture_output=True, text=True)

    def ask(m, n, k, mats, terms):
        r = subprocess.run([str(exe)], input=f"{m} {n} {k} {mats} {terms}\n", capture_output=True, text=True, check=True)
        kind, tm, dx, dx_splits, dw, dw_splits = r.stdout.split()
        return f"{kind} {tm}", (dx, int(dx_splits)), (dw, int(dw_splits))

    return ask


@pytest.mark.parametrize("shape", list(GATED))
def test_gated_shapes_reach_their_kernels(plan, shape):
    kernel, dx, dw = GATED[shape]
    assert [plan(*shape, 2, t) for t in (1, 2, 3)] == [(kernel, dx[t], dw[t]) for t in range(3)]


@pytest.mark.parametrize("shape", list(LINEAR))
def test_linear_shapes_reach_their_kernels(plan, shape):
    dx, dw = LINEAR[shape]
    assert [plan(*shape, 1, t)[1:] for t in (1, 2, 3)] == [(dx[t], dw[t]) for t in range(3)]


def test_every_kernel_of_the_gated_block_is_reached():
    assert {v[0] for v in GATED.values()} == {"split 1", "split 2", "gemm 1", "gemm 2", "gemm 3", "gemm 4"}
    for terms in range(3):
        dx = {(tile, splits > 1) for tile, splits in (v[1][terms] for v in GATED.values())}
        assert dx == {(tile, s) for tile in ("128x64", "256x64", "256x256") for s in (False, True)}
        assert {v[2][terms][0] for v in GATED.values()} == {"256x64", "256x256"}
    assert {(v[2][t][0], v[2][t][1] > 1) for v in GATED.values() for t in range(3)} == {
        (tile, s) for tile in ("256x64", "256x256") for s in (False, True)}
