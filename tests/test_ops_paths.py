"""Which kernels the operators' rules pick, on the CPU: the sizes of ops_paths.py, which
the GPU tests run, lead where their names say (tests/native/ops_plan_show.cpp prints
the plans)."""
import os
import shutil
import subprocess

import pytest

import ops_paths

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2411_17866_amd", "csrc")
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def show(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    if not os.path.exists(os.path.join(ROCM_INCLUDE, "hip", "hip_runtime_api.h")):
        pytest.skip("HIP headers not installed")
    exe = str(tmp_path_factory.mktemp("plans") / "ops_plan_show")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Wextra", "-Wno-unused-parameter", "-D__HIP_PLATFORM_AMD__",
                        f"-I{ROCM_INCLUDE}", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "native", "ops_plan_show.cpp"),
                        os.path.join(CSRC, "ops_runtime.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]

    def run(*problems):
        r = subprocess.run([exe, *(",".join(map(str, p)) for p in problems)], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return [line.split() for line in r.stdout.splitlines()]

    return run


def _ce(show, size, dtype, grads):
    form, *numbers = show((*size, dtype, grads))[0]
    return form, dict(zip(("tile", "columns", "front", "pieces", "splits", "sample"), map(int, numbers)))


@pytest.mark.parametrize("size,want", ops_paths.GRADIENTS, ids=str)
def test_gradients_by_tiles_of_256(show, size, want):
    for dtype in (F32, BF16):
        form, q = _ce(show, size, dtype, 1)
        assert form == ("halves", "half")[dtype] and q["tile"] == 256
        assert (q["sample"] > 0) == want["refs"]
        assert q["pieces"] == want.get("pieces", (1, 1))[dtype]


@pytest.mark.parametrize("size,want", ops_paths.LOSSES, ids=str)
def test_losses_by_tiles_of_256(show, size, want):
    for dtype in (F32, BF16):
        form, q = _ce(show, size, dtype, 0)
        assert form == ("halves", "bf16")[dtype] and q["tile"] == 256
        assert (q["front"] < q["columns"]) == want["split"]


@pytest.mark.parametrize("shape,want", ops_paths.MATRICES, ids=str)
def test_matrices(show, shape, want):
    count, rows, cols = shape
    assert tuple(map(int, show(("ortho", count, rows, cols))[0])) == (0, *want)
