"""The host runtime of the linear layer, the norms and clipping on the CPU: plans,
argument checks and launch arguments under AddressSanitizer and UBSan
(tests/native/block_host_check.cpp); where the rules lead the sizes of block_paths.py
(tests/native/block_plan_show.cpp); and the library's refusals through the binding."""
import ctypes
import os
import shutil
import subprocess

import pytest

import block_paths
from paper_2411_17866_amd import dsm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2411_17866_amd", "csrc")
RUNTIME = os.path.join(CSRC, "block_runtime.cpp")
ROCM_INCLUDE = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
SANITIZED = ("-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan")
F32, BF16 = dsm.DSM_F32, dsm.DSM_BF16


def _build(folder, check, runtime, *flags):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    if not os.path.exists(os.path.join(ROCM_INCLUDE, "hip", "hip_runtime_api.h")):
        pytest.skip("HIP headers not installed")
    exe = str(folder / check)
    # Host code only: g++, no HIP source on this line.
    r = subprocess.run([gxx, "-std=c++17", "-O1", *flags, "-Wall", "-Wextra", "-Wno-unused-parameter", "-D__HIP_PLATFORM_AMD__",
                        f"-I{ROCM_INCLUDE}", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "native", check + ".cpp"), runtime, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def _check(folder, runtime, *flags):
    exe = _build(folder, "block_host_check", runtime, *flags)
    return subprocess.run([exe], capture_output=True, text=True, timeout=600)


def test_runtime_under_sanitizers(tmp_path):
    r = _check(tmp_path, RUNTIME, *SANITIZED)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "all checks passed" in r.stdout


@pytest.mark.parametrize("planted", [
    ("q.y_parts = take(q.splits > 1 ? q.splits * T * q.ld_y * 4 : 0);", "q.y_parts = take(T * q.ld_y * 4);"),
    ("(p->grads && q.dz_halves ? 2 * q.pad_tokens : T)", "T"),
    ("q.ld_dim = round_up(D, 64) * width;", "q.ld_dim = round_up(D, 32) * width;"),
    ("q.dz = take(q.pad_tokens * q.ld_wide * (q.dz_halves ? 4 : 2));", "q.dz = take(T * q.ld_wide * (q.dz_halves ? 4 : 2));"),
    ("q.bias_sums = take(q.bias_parts * N * 4);", "q.bias_sums = take(q.bias_parts * N * 2);"),
    ("q.dw_splits * N * q.ld_dx * 4", "q.dw_splits * N * D * 4"),
    ("q.tops = take(q.pad_tokens / q.split_rows * 4);", "q.tops = take(q.pad_tokens / 8 * 4);"),
    ("T >= 1536 || N > 8192 ? 8 : 2", "T >= 1536 ? 8 : 2"),
    ("p.tokens % 64 == 0));", "true));"),
    ("(c.p.back_few || (direct", "((direct"),
    ("q.back_few = T <= (q.f32 ? kSingleBackward : kFewBackward);", "q.back_few = T <= kSingleBackward;"),
    ("!c.p.dz_halves && direct", "direct"),
    ("stride * size < kMaxStride * 2 && ", ""),
    ("if (form == dsm::kLinearHalves) return false;", ""),
    ("o.dw_dtype == p->dw_dtype && ", ""),
    ("std::copy(sums, sums + dsm::kNormSums, c.sums);", "std::copy(sums, sums + 4, c.sums);"),
    ("if (!needs_f) c.f = nullptr;", "c.f = nullptr;"),
    ("e->group != next.group || ", ""),
    (" || e->bf16 != next.bf16", ""),
    ("|| e->first + e->numel != next.first", ""),
    ("table->slot += table->chunks;", ""),
    ("if (table->count == dsm::kClipEntries) break;", "if (table->count == dsm::kClipEntries - 1) { ++*i; break; }"),
    ("scales && launches == 1 && ", "scales && "),
    ("groups.start[g + 1] = groups.start[g] + counts[g];", "groups.start[g + 1] = counts[g];"),
])
def test_planted_mistakes_fail_the_host_checks(tmp_path, planted):
    with open(RUNTIME) as f:
        source = f.read()
    assert source.count(planted[0]) == 1, planted[0]
    copy = tmp_path / "block_runtime.cpp"
    copy.write_text(source.replace(*planted))
    assert _check(tmp_path, str(copy)).returncode != 0


@pytest.fixture(scope="module")
def show(tmp_path_factory):
    exe = _build(tmp_path_factory.mktemp("plans"), "block_plan_show", RUNTIME)

    def plan(*problem):
        r = subprocess.run([exe, ",".join(map(str, problem))], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        words = r.stdout.split()
        return dict(zip(words[::2], words[1::2]))

    return plan


@pytest.mark.parametrize("size,f32,bf16", block_paths.FORWARD, ids=str)
def test_forward_paths(show, size, f32, bf16):
    for dtype, want in ((F32, f32), (BF16, bf16)):
        assert block_paths.forward_way(size, show(*size, dtype, dsm.DSM_ACT_SILU, dtype)) == want


@pytest.mark.parametrize("size,f32,bf16,mixed", block_paths.BACKWARD, ids=str)
def test_backward_paths(show, size, f32, bf16, mixed):
    for dtype, dw, want in ((F32, F32, f32), (BF16, BF16, bf16), (BF16, F32, mixed)):
        assert block_paths.backward_way(size, show(*size, dtype, dsm.DSM_ACT_SILU, dw)) == want


def test_every_tile_and_part_is_among_the_paths():
    forward = {w for _, *ways in block_paths.FORWARD for w in ways}
    assert {f"few {g} parts" for g in (1, 2, 4)} | {"single 64", "single 64 parts", "halves 128 parts", "bf16 128 parts", "halves 256",
                                                    "halves 256 front", "halves 256 parts", "bf16 64", "bf16 256", "bf16 256 front"} <= forward
    for kind in range(3):
        ways = {w[kind] for _, *w in block_paths.BACKWARD}
        assert {"64 dx dw", "128 dx dw", "256 dw", "256 dx dw"} & ways >= ({"128 dx dw", "256 dw", "256 dx dw"})


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(tokens=2 ** 20 + 1), dict(dim=0), dict(wide=2 ** 16 + 1), dict(dtype=2),
                                 dict(act=9), dict(dw_dtype=BF16), dict(grads=-1)], ids=str)
def test_linear_problems(bad):
    good = dict(tokens=100, dim=64, wide=80, dtype=F32, act=dsm.DSM_ACT_GELU, dw_dtype=F32, grads=1)
    assert dsm.dsm_linear_workspace(dsm.dsm_linear_problem(**good)) > 0
    problem = dsm.dsm_linear_problem(**dict(good, **bad))
    for call in (lambda: dsm.dsm_linear_workspace(problem), lambda: dsm.dsm_linear(problem, dsm.dsm_linear_buffers()),
                 lambda: dsm.dsm_linear_backward(problem, dsm.dsm_linear_buffers())):
        with pytest.raises(dsm.DsmError) as e:
            call()
        assert e.value.status == dsm.DSM_ERR_INVALID_ARG
        assert dsm.dsm_last_error(None) == e.value.message


@pytest.mark.parametrize("bad", [dict(tokens=-1), dict(dim=8193), dict(dtype=-1), dict(norm=3), dict(post=4), dict(grads=2), dict(eps=-1.0),
                                 dict(post_eps=float("nan")), dict(scale=float("inf"))], ids=str)
def test_norm_problems(bad):
    good = dict(tokens=100, dim=64, dtype=BF16, norm=dsm.DSM_NORM_RMS, post=dsm.DSM_NORM_NONE, grads=1, eps=1e-5, post_eps=1e-5, scale=1.0)
    assert dsm.dsm_norm_workspace(dsm.dsm_norm_problem(**good)) > 0
    problem = dsm.dsm_norm_problem(**dict(good, **bad))
    for call in (lambda: dsm.dsm_norm_workspace(problem), lambda: dsm.dsm_residual_norm(problem, dsm.dsm_norm_buffers()),
                 lambda: dsm.dsm_residual_norm_backward(problem, dsm.dsm_norm_buffers())):
        with pytest.raises(dsm.DsmError) as e:
            call()
        assert e.value.status == dsm.DSM_ERR_INVALID_ARG


def test_clip_tensors():
    one = (dsm.dsm_clip_tensor * 1)(dsm.dsm_clip_tensor(0, 0, 100, 100, 100, F32, 0))
    assert dsm.dsm_clip_workspace(one, 1) > 0
    for n_groups in (0, 257):
        with pytest.raises(dsm.DsmError):
            dsm.dsm_clip_workspace(one, n_groups)
    for field, value in (("numel", -1), ("block", 0), ("stride", 99), ("dtype", 2), ("group", 1), ("first", -1)):
        bad = (dsm.dsm_clip_tensor * 1)(dsm.dsm_clip_tensor(0, 0, 100, 100, 100, F32, 0))
        setattr(bad[0], field, value)
        with pytest.raises(dsm.DsmError):
            dsm.dsm_clip_workspace(bad, 1)
    with pytest.raises(dsm.DsmError) as e:  # data is NULL
        dsm.dsm_grad_clip(one, 1, 1.0, 256, 256, 1 << 20, 1e-6, 0)
    assert "NULL" in e.value.message


def test_sizes_of_the_structures():
    """The binding's structures have the header's fields: words of 8 bytes, and of 4 in pairs."""
    assert ctypes.sizeof(dsm.dsm_linear_problem) == 3 * 8 + 4 * 4
    assert ctypes.sizeof(dsm.dsm_linear_buffers) == 21 * 8
    assert ctypes.sizeof(dsm.dsm_norm_problem) == 2 * 8 + 7 * 4 + 4
    assert ctypes.sizeof(dsm.dsm_norm_buffers) == (8 * 2 + 10 + 3) * 8
    assert ctypes.sizeof(dsm.dsm_clip_tensor) == 5 * 8 + 2 * 4


def test_no_plan_without_a_gpu():
    ops = pytest.importorskip("paper_2411_17866_amd.ops")
    for make in (lambda: ops.Linear(4, 8, 8, device="cpu"), lambda: ops.ResidualNorm(4, 8, device="cpu"),
                 lambda: ops.GradClip([], device="cpu"), lambda: ops.Linear(4, 8, 8, act="swish", device="cpu"),
                 lambda: ops.ResidualNorm(4, 8, norm="batch", device="cpu")):
        with pytest.raises(ValueError):
            make()
