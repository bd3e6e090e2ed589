"""What the kernels of the linear layer, the norms and clipping promise the compiler about the addresses of
rows, which may start at any element: 16-byte loads and stores of the caller's rows promise the alignment of
one element, 2 bytes of bf16, 4 of fp32.  (The device's own assembly would not tell: it has one instruction
for all.)  Only copies in the workspace are known to lie on 16 bytes."""
import collections
import os
import re
import subprocess

import pytest

from paper_2411_17866_amd import build
from test_ops_isa import pytestmark  # noqa: F401

SIZES = {"i16": 2, "half": 2, "bfloat": 2, "i32": 4, "float": 4, "i64": 8, "double": 8}
# Kernels that read or write fp32 dz or fp16 halves in the workspace by 16 bytes.
OWN = re.compile(r"k_few_backwardILi|k_dz_split|k_back_copies|k_copiesILNS_10LinearFormE1")


@pytest.fixture(scope="module")
def accesses(tmp_path_factory):
    folder = tmp_path_factory.mktemp("ir")

    def of(source):
        """kernel -> Counter of (bytes of an element, bytes, alignment) of global vector loads and stores."""
        out = str(folder / (source + ".ll"))
        r = subprocess.run([build.hipcc(), "-x", "hip", *build.COMMON_FLAGS, *build.DEVICE_FLAGS, "--offload-device-only", "-S",
                            "-emit-llvm", os.path.join(build.CSRC, source), "-o", out], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
        seen, name = collections.defaultdict(collections.Counter), None
        with open(out) as f:
            for line in f:
                m = re.match(r"define .*@(\S+?)\(", line)
                if m:
                    name = m.group(1)
                m = re.search(r"(?:= load|\bstore) <(\d+) x (\w+)>[^@]*ptr addrspace\(1\).*align (\d+)", line)
                if m and name:
                    each = SIZES[m.group(2)]
                    seen[name][each, each * int(m.group(1)), int(m.group(3))] += 1
        return seen

    return of


@pytest.mark.parametrize("source,least", [("norm.hip", 500), ("clip.hip", 20), ("linear.hip", 500)])
def test_rows_may_start_at_any_element(accesses, source, least):
    bad, seen = {}, 0
    for kernel, counts in accesses(source).items():
        for (each, size, align), n in counts.items():
            if size < 8:
                continue
            seen += n
            if align > 4 and not OWN.search(kernel):
                bad[kernel] = counts
    assert not bad, bad
    assert seen >= least, seen


def test_bf16_rows_of_few_tokens(accesses):
    """Their runs are turned as fours of floats: of an element's alignment all the same.  (Two loads of 16 bytes at
    fp32's alignment are the bias's, two stores those of a part of the sums.)"""
    few = {k: v for k, v in accesses("linear.hip").items() if "5k_fewILb0E" in k}
    assert len(few) == 3
    for kernel, counts in few.items():
        loose = sum(n for (_, size, align), n in counts.items() if size == 16 and align == 2)
        fp32 = sum(n for (_, size, align), n in counts.items() if size == 16 and align == 4)
        groups = int(re.search(r"k_fewILb0ELi(\d)", kernel).group(1))
        assert loose >= (2 if groups < 4 else 1) * 2 * (1 + groups), (kernel, counts)
        assert fp32 <= 4, (kernel, counts)
