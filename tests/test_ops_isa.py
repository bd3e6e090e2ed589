"""The operators' compiled kernels by tiles of up to 128, and those without tiles: at every
barrier a wave's reads and writes of LDS are done, along every path to it.  Behind the
barrier other waves overwrite what was read, and in the source of these tiles only the use
of a value, not a wait of its own, says that a read is over (an explicit wait costs a
single token's loss 4%).  Tiles of 256 wait in their source, by branches whose conditions
this look at paths does not follow."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2411_17866_amd import build

pytestmark = pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                                reason="no hipcc")


def kernels(assembly):
    """name -> [(label or None, instruction)] of each function."""
    out, name = {}, None
    for line in assembly.splitlines():
        text = line.split(";")[0].strip()
        m = re.match(r"^([A-Za-z_.$][\w.$]*):$", text)
        if m and m.group(1).startswith("_Z"):
            name = out.setdefault(m.group(1), [])
        elif m and name is not None:
            name.append((m.group(1), None))
        elif text.startswith(".Lfunc_end") or text.startswith(".section"):
            name = None
        elif name is not None and text and not text.startswith("."):
            name.append((None, text))
    return out


def unfinished(code):
    """Barriers that some path reaches with LDS accesses in flight, of all barriers."""
    blocks, labels = [[]], {}
    for label, text in code:
        if label is not None:
            if blocks[-1]:
                blocks.append([])
            labels[label] = len(blocks) - 1
            continue
        blocks[-1].append(text)
        if re.match(r"s_(cbranch|branch|endpgm|setpc)", text):
            blocks.append([])
    entry, todo = {0: 0}, [0]
    found, seen = set(), set()
    while todo:
        b = todo.pop()
        flying, falls, targets = entry[b], True, []
        for k, text in enumerate(blocks[b]):
            op = text.split()[0]
            if op.startswith("ds_"):
                flying = min(flying + 1, 15)
            elif op == "s_waitcnt":
                m = re.search(r"lgkmcnt\((\d+)\)", text)
                if m:
                    flying = min(flying, int(m.group(1)))
            elif op == "s_barrier":
                seen.add((b, k))
                if flying:
                    found.add((b, k))
            elif op.startswith("s_cbranch") or op == "s_branch":
                targets.append(labels[text.split()[-1]])
                falls = op != "s_branch"
            elif op in ("s_endpgm", "s_setpc_b64"):
                falls = False
        for t in targets + ([b + 1] if falls and b + 1 < len(blocks) else []):
            if flying > entry.get(t, -1):
                entry[t] = flying
                todo.append(t)
    return len(found), len(seen)


def test_the_check_sees_a_missing_wait():
    loop = [(None, "s_waitcnt lgkmcnt(0)"), (".L1", None), (None, "s_barrier"), (None, "ds_read_b128 v[0:3], v4"),
            (None, "s_waitcnt lgkmcnt(0)"), (None, "s_cbranch_scc1 .L1"), (None, "s_barrier"), (None, "s_endpgm")]
    assert unfinished(loop) == (0, 2)
    assert unfinished(loop[:4] + loop[5:]) == (2, 2)  # along the back edge, and behind the loop
    late = loop[:4] + [(None, "ds_read_b128 v[5:8], v9"), (None, "s_waitcnt vmcnt(0) lgkmcnt(1)")] + loop[5:]
    assert unfinished(late) == (2, 2)


@pytest.mark.parametrize("source", ["linear_ce.hip", "ortho.hip"])
def test_lds_accesses_end_before_a_barrier(source, tmp_path):
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
    assert barriers > 100
