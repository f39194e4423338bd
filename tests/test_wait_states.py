"""The wait states that gfx9 leaves to the program, in the built kernels (CPU: the library's
device code is disassembled).  The compiler keeps them in what it writes itself, but does not
look into inline assembly:

* a scalar write of m0, then a load to LDS (which takes its address from m0): 1;
* a vector instruction that writes scalar registers, then a memory instruction that reads
  them: 5.

Every instruction counts as one wait state, s_nop n as n + 1.
"""

import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_04244_amd import build

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
M0_BEFORE_LDS_LOAD, SGPR_BEFORE_MEMORY = 1, 5
MEMORY = ("global_", "buffer_", "flat_", "scratch_")


def scalars(operand):
    """The scalar registers an operand names: numbers, and "vcc" for both halves."""
    m = re.fullmatch(r"s(\d+)|s\[(\d+):(\d+)\]", operand)
    if m:
        return {int(m.group(1))} if m.group(1) else set(range(int(m.group(2)), int(m.group(3)) + 1))
    return {"vcc"} if operand.startswith("vcc") else set()


def violations(lines):
    """[(function, instruction, what is missing)] of a disassembly."""
    bad, name, m0, written = [], "", None, {}          # wait states since the writes
    for line in lines:
        head = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if head:
            name, m0, written = head.group(1), None, {}
            continue
        text = line.split("//")[0].strip()
        if not re.match(r"[a-z]+_\w+", text):
            continue
        op, _, rest = text.partition(" ")
        words = re.findall(r"s\[\d+:\d+\]|[\w\[\]:.-]+", rest)
        if op.startswith(MEMORY):
            if ("_lds_" in op or "lds" in words) and m0 is not None and m0 < M0_BEFORE_LDS_LOAD:
                bad.append((name, text, "m0"))
            for r in set().union(*(scalars(w) for w in words)):
                if written.get(r, SGPR_BEFORE_MEMORY) < SGPR_BEFORE_MEMORY:
                    bad.append((name, text, f"scalar {r}"))
        passed = int(words[0], 0) + 1 if op == "s_nop" else 1
        m0 = None if m0 is None else m0 + passed
        written = {r: n + passed for r, n in written.items() if n + passed < SGPR_BEFORE_MEMORY}
        if words and op.startswith("s_"):
            if words[0] == "m0" and not op.startswith("s_cmp"):
                m0 = 0
            for r in scalars(words[0]):                 # a scalar write replaces the vector one
                written.pop(r, None)
        elif op.startswith("v_"):
            for w in words[:2] if "_co_" in op or op.startswith("v_div_scale") else words[:1]:
                written.update({r: 0 for r in scalars(w)})
    return bad


def test_the_check_itself():
    m0 = ["0000 <f>:", "\ts_mov_b32 m0, s3", "\tglobal_load_lds_dwordx4 v[0:1], off // 0"]
    assert len(violations(m0)) == 1 and not violations(m0[:2] + ["\ts_nop 0"] + m0[2:])
    assert violations(["0 <f>:", "\ts_add_u32 m0, s3, 16", "\tbuffer_load_dword v0, s[0:3], s4 offen lds"])
    lane = ["0 <f>:", "\tv_readfirstlane_b32 s4, v9"]
    load = ["\tglobal_load_dwordx4 v[0:3], v9, s[4:5]"]
    for waits, ok in (([], False), (["\ts_nop 3"], False), (["\ts_nop 4"], True), (["\tv_mov_b32_e32 v0, 1"] * 5, True)):
        assert (violations(lane + waits + load) == []) == ok
    assert not violations(lane + ["\ts_mov_b32 s4, s8"] + load) and not violations(lane + ["\tglobal_load_dword v0, v9, s[6:7]"])


def test_built_kernels_keep_the_wait_states(tmp_path):
    if not (os.path.exists(OBJDUMP) and os.path.exists(build.LIB)):
        pytest.skip("needs llvm-objdump and a built library")
    lib = shutil.copy(build.LIB, tmp_path / "libqlin.so")
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True, timeout=300)
    parts = glob.glob(str(tmp_path / f"*amdgcn*{build.ARCH}*"))
    assert parts
    loads, bad = 0, []
    for part in parts:
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", part], check=True, capture_output=True, text=True, timeout=600).stdout
        loads += len(re.findall(r"load_lds_|\blds$", text.replace(" //", "\n//"), re.M))
        bad += violations(text.splitlines())
    assert loads > 100                                   # the kernels that load to LDS are there
    assert not bad, f"{len(bad)}: {bad[:5]}"
