"""The compiled kernels of the linear layer, the norms and clipping: at every barrier a
wave's reads and writes of LDS are done, along every path to it (tiles of 256, which wait
in their source, aside)."""
import os
import subprocess

import pytest

from paper_2411_17866_amd import build
from test_ops_isa import kernels, pytestmark, unfinished  # noqa: F401


@pytest.mark.parametrize("source,least", [("linear.hip", 60), ("norm.hip", 60), ("clip.hip", 3)])
def test_lds_accesses_end_before_a_barrier(source, least, tmp_path):
    out = str(tmp_path / "kernels.s")
    r = subprocess.run([build.hipcc(), "-x", "hip", *build.COMMON_FLAGS, *build.DEVICE_FLAGS, "--offload-device-only", "-S",
                        os.path.join(build.CSRC, source), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    with open(out) as f:
        code = kernels(f.read())
    barriers = 0
    for name, body in code.items():
        if "Li256E" in name:
            continue
        bad, all_ = unfinished(body)
        barriers += all_
        assert bad == 0, f"{name}: {bad} of {all_} barriers"
    assert barriers >= least, barriers
