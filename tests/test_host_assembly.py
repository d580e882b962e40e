"""The instructions of the built kernels: what the hardware asks for around loads from memory to LDS, which are written by hand
(the compiler looks after its own instructions, not into inline assembly)."""
import collections
import os
import re
import shutil
import subprocess

import pytest

import paper_1905_10138_amd as xe

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
BEFORE = 8  # instructions kept before each


@pytest.fixture(scope="module")
def loads_to_lds(tmp_path_factory):
    """(kernel, the instructions before, the load) of every load from memory to LDS, and every other instruction that names m0."""
    if OBJDUMP is None:
        pytest.skip("no llvm-objdump here")
    there = tmp_path_factory.mktemp("kernels")
    library = shutil.copy(xe.library_path(), there)
    subprocess.run([OBJDUMP, "--offloading", library], check=True, capture_output=True, timeout=60)
    parts = sorted(str(p) for p in there.iterdir() if p.name.endswith("gfx950"))
    assert len(parts) >= 10
    loads, others, kernel, last = [], collections.Counter(), "", collections.deque(maxlen=BEFORE)
    with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", *parts], stdout=subprocess.PIPE, text=True) as dump:
        for line in dump.stdout:
            if line.endswith(">:\n"):
                kernel = line.split("<")[1][:-3]
                last.clear()
                continue
            if not line.startswith("\t"):
                continue
            text = line.split("//")[0].strip()
            if text.startswith("buffer_load") and text.endswith(" lds"):
                loads.append((kernel, tuple(last), text))
            elif "m0" in text and not text.startswith("s_mov_b32 m0, s"):
                others[text] += 1
            last.append(text)
    assert dump.returncode == 0
    return loads, others


def test_loads_to_lds_wait_for_m0(loads_to_lds):
    # a load to LDS takes its place from m0, and needs an instruction (or a wait state) between the one that writes m0 and itself
    loads, others = loads_to_lds
    assert len({kernel for kernel, _, _ in loads}) > 300
    short = {kernel for kernel, before, _ in loads if re.match(r"s_\w+ m0,", before[-1])}
    assert not short
    assert not others  # and nothing else has a value of its own there


def wait_states(text):
    m = re.match(r"s_nop (\d+)", text)
    return 1 + int(m[1]) if m else 1


def registers(operand):
    m = re.match(r"s\[(\d+):(\d+)\]$|s(\d+)$", operand)
    return set() if not m else set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}


def test_loads_to_lds_wait_for_their_scalar_operands(loads_to_lds):
    # five wait states between a vector instruction that writes a scalar register and a load that reads it: what stands before a load
    # in those five is its own two instructions, or nothing that writes them (a jump ends what can be seen, and counts as a write)
    loads, _ = loads_to_lds
    short = set()
    for kernel, before, load in loads:
        needed = set().union(*(registers(operand.split()[0]) for operand in load.split(None, 1)[1].split(",")[1:]))
        assert len(needed) >= 4
        left = 5
        for text in reversed(before):
            if left <= 0:
                break
            operands = text.split(None, 1)[1].split(",") if " " in text else []
            writes = set().union(*(registers(o.strip()) for o in operands[:2])) if text.startswith("v_") else set()
            if writes & needed or "branch" in text:
                short.add((kernel, text, load))
                break
            left -= wait_states(text)
        else:
            if left > 0:
                short.add((kernel, "", load))
    assert not short
