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
