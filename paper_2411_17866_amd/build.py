"""Builds libdsm.so (the C-ABI library of include/dsm.h) for gfx950 with hipcc.

    python -m paper_2411_17866_amd.build

Output: paper_2411_17866_amd/lib/libdsm.so.  Intermediate objects go to
_build/ at the repository root.  Every call compiles from source.
"""
import os
import shutil
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

PKG = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(PKG)
CSRC = os.path.join(PKG, "csrc")
INCLUDE = os.path.join(ROOT, "include")
LIBDIR = os.path.join(PKG, "lib")
OBJDIR = os.path.join(ROOT, "_build")
LIBPATH = os.path.join(LIBDIR, "libdsm.so")

ARCH = "gfx950"
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

KERNELS = ["dsm_kernels.hip", "ortho.hip", "linear_ce.hip", "linear.hip", "norm.hip", "clip.hip"]
HOST = ["dsm_runtime.cpp", "ops_runtime.cpp", "block_runtime.cpp"]

# Numerics: one IEEE fp32 rounding per written operation (no FMA contraction),
# correctly rounded division and square root, denormals kept.  Packed fp32
# instructions are disabled.
COMMON_FLAGS = [
    "-O3", "-std=c++17", "-fPIC", "-fvisibility=hidden", "-Wall", "-Wextra",
    "-Wno-unused-parameter",
    "-ffp-contract=off",
    f"-I{INCLUDE}", f"-I{CSRC}",
]
DEVICE_FLAGS = [
    f"--offload-arch={ARCH}",
    "-fno-gpu-flush-denormals-to-zero",
    "-fhip-fp32-correctly-rounded-divide-sqrt",
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
]


def hipcc():
    exe = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(exe):
        raise RuntimeError("hipcc not found; the library needs ROCm's hipcc to build")
    return exe


def _run(cmd, verbose):
    if verbose:
        print(" ".join(cmd), flush=True)
    r = subprocess.run(cmd, capture_output=True, text=True)
    if r.returncode != 0:
        raise RuntimeError(f"command failed ({r.returncode}): {' '.join(cmd)}\n{r.stdout}\n{r.stderr}")
    return r


def build(verbose=False, out=LIBPATH):
    """Compiles the kernels and the host runtime and links libdsm.so."""
    os.makedirs(os.path.dirname(out), exist_ok=True)
    objdir = os.path.join(OBJDIR, "default")
    os.makedirs(objdir, exist_ok=True)
    cc = hipcc()
    objs = [os.path.join(objdir, os.path.splitext(src)[0] + ".o") for src in KERNELS + HOST]

    def compile_one(job):
        src, obj = job
        lang = (["-x", "hip", *COMMON_FLAGS, *DEVICE_FLAGS] if src in KERNELS else
                ["-x", "c++", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", *COMMON_FLAGS])
        _run([cc, *lang, "-c", os.path.join(CSRC, src), "-o", obj], verbose)

    with ThreadPoolExecutor(max_workers=len(objs)) as pool:
        list(pool.map(compile_one, zip(KERNELS + HOST, objs)))
    tmp = out + ".tmp"
    _run([cc, "-shared", f"--offload-arch={ARCH}", "-o", tmp, *objs,
          "-Wl,--no-undefined", "-Wl,-soname,libdsm.so"], verbose)
    os.replace(tmp, out)
    return out


def kernel_isa(path=None):
    """Writes the gfx950 assembly of the kernels, compiled with the library's flags, for review."""
    out = path or os.path.join(OBJDIR, "dsm_kernels.s")
    _run([hipcc(), "-x", "hip", *COMMON_FLAGS, *DEVICE_FLAGS, "--offload-device-only", "-S",
          os.path.join(CSRC, "dsm_kernels.hip"), "-o", out], False)
    return out


if __name__ == "__main__":
    print(build(verbose="-v" in sys.argv))
