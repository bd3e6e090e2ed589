"""The operators' host runtime on the CPU: plans, argument checks and launch
arguments under AddressSanitizer and UBSan (tests/native/ops_host_check.cpp), and the
library's refusals through the binding."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2411_17866_amd import dsm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2411_17866_amd", "csrc")
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")


def _build(tmp_path, source):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    if not os.path.exists(os.path.join(ROCM_INCLUDE, "hip", "hip_runtime_api.h")):
        pytest.skip("HIP headers not installed")
    exe = str(tmp_path / "ops_host_check")
    # Host code only: g++, no HIP source on this line.
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
           "-Wall", "-Wextra", "-Wno-unused-parameter",
           "-D__HIP_PLATFORM_AMD__", f"-I{ROCM_INCLUDE}", f"-I{os.path.join(ROOT, 'include')}",
           f"-I{CSRC}", os.path.join(ROOT, "tests", "native", "ops_host_check.cpp"), source,
           "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return subprocess.run([exe], capture_output=True, text=True, timeout=600)


def test_operators_runtime_under_sanitizers(tmp_path):
    r = _build(tmp_path, os.path.join(CSRC, "ops_runtime.cpp"))
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout


@pytest.mark.parametrize("planted", [
    ("q.h = take(tokens_pad * q.ld_h * 2);", "q.h = take(T * q.ld_h * 2);"),
    ("q.ld_h = q.ld_w = round_up(p->dim, 64) * width;", "q.ld_h = q.ld_w = round_up(p->dim, 32) * width;"),
    ("q.dh = take(q.dh_splits * T * q.ld_dh * 4);", "q.dh = take(T * q.ld_dh * 4);"),
    ("(q.form == dsm::kCeBf16 ? 4 : 2)", "2"),
    ("b.w_stride * elem % 16 == 0 && aligned(b.w, 16)", "aligned(b.w, 16)"),
    ("!p.grads && b.h_stride", "b.h_stride"),
    ("s.b = exponent_under(top_b * 1.01);", "s.b = exponent_under(l);"),
    ("if (k > 0) it->scales[k - 1].x_next = s.x;", ""),
    ("g.off.at[i] = p->offsets[first + i];", "g.off.at[i] = p->offsets[i];"),
    ("vector = vector && p->offsets[i] % 4 == 0;", ""),
])
def test_planted_mistakes_fail_the_host_checks(tmp_path, planted):
    source = open(os.path.join(CSRC, "ops_runtime.cpp")).read()
    assert source.count(planted[0]) == 1, planted[0]
    copy = tmp_path / "ops_runtime.cpp"
    copy.write_text(source.replace(*planted))
    assert _build(tmp_path, str(copy)).returncode != 0


def test_refusals_through_the_binding():
    if not os.path.exists(dsm.LIBPATH):
        from paper_2411_17866_amd import build
        build.build()
    assert dsm.dsm_ce_workspace(dsm.dsm_ce_problem(100, 64, 1000, dsm.DSM_F32, 1)) > 0
    for bad in ((-1, 64, 10, 0, 0), (1, 0, 10, 0, 0), (1, 64, 0, 0, 0), (1, 64, 10, 2, 0), (1, 64, 10, 0, 3)):
        with pytest.raises(dsm.DsmError) as e:
            dsm.dsm_ce_workspace(dsm.dsm_ce_problem(*bad))
        assert e.value.status == dsm.DSM_ERR_INVALID_ARG
        assert dsm.dsm_last_error(None) == e.value.message
    assert dsm.dsm_ortho_workspace(dsm.make_ortho_problem(64, 48, [0])) == 0
    assert dsm.dsm_ortho_workspace(dsm.make_ortho_problem(768, 2304, [0] * 12)) > 0
    with pytest.raises(dsm.DsmError):
        dsm.dsm_orthogonalize(dsm.make_ortho_problem(768, 64, [0]), dsm.dsm_ortho_buffers())
    with pytest.raises(dsm.DsmError):
        dsm.dsm_ortho_step(dsm.make_ortho_problem(8, 8, [0], dtype=dsm.DSM_BF16),
                           dsm.dsm_ortho_buffers(), 0.1, 0.9)
    with pytest.raises(ValueError):
        dsm.make_ortho_problem(8, 8, [0], steps=2, coeffs=[[1, 0, 0]])
    lib = dsm.load_library()
    assert lib.dsm_linear_ce(None, None, 0) == dsm.DSM_ERR_INVALID_ARG
    assert lib.dsm_ortho_workspace(None, ctypes.byref(ctypes.c_int64())) == dsm.DSM_ERR_INVALID_ARG
