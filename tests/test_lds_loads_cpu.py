"""Waits that the built kernels owe the hardware around their direct global->LDS loads, read from the library's own code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2411_01171_amd.build import LIB_PATH

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"
SCALAR = re.compile(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)")


def _scalars(operand):
    """Scalar registers that an operand names."""
    if operand.startswith("vcc"):
        return {"vcc"}
    m = SCALAR.match(operand)
    if not m:
        return set()
    return {int(m[3])} if m[3] else set(range(int(m[1]), int(m[2]) + 1))


def _states(text):
    """Wait states that an instruction stands for."""
    return int(text.split()[1], 0) + 1 if text.startswith("s_nop") else 1


def owed(listing):
    """(loads, waits missing) of a disassembly: one state between a scalar write of M0 and a load to LDS, five between a vector
    instruction's write of a scalar register and a load that takes its address from it.  An instruction that uses M0 for
    something else is listed with them: the loads' assembly changes M0 behind the compiler's back."""
    loads, missing, before = 0, [], []  # before: the instructions in front, nearest last
    for line in listing:
        if line.endswith(">:\n"):
            before = []
            continue
        text = line.split("//")[0].strip()
        if not text or text.endswith(":") or text.startswith("/"):
            continue
        op, _, rest = text.partition(" ")
        operands = [t.strip() for t in rest.split(",")]
        if "m0" in rest and not text.startswith("s_mov_b32 m0, "):
            missing.append((text, "M0"))
        if "load_lds_" in op or (op.startswith("buffer_load") and re.search(r"\blds\b", rest)):
            loads += 1
            reads, states = set().union(*(_scalars(t) for t in operands)), 0
            for earlier, written in reversed(before):
                if states < 1 and earlier.startswith("s_") and "m0" in written:
                    missing.append((earlier, text))
                if states < 5 and earlier.startswith("v_") and written & reads:
                    missing.append((earlier, text))
                states += _states(earlier)
        written = {"m0"} if operands[0] == "m0" else _scalars(operands[0])
        if "_co_" in op and len(operands) > 1:  # the carry
            written = written | _scalars(operands[1])
        before = before[-5:] + [(text, written)]
    return loads, missing


def test_the_count_itself():
    listing = ["k>:\n", "\ts_mov_b32 m0, s4\n", "\tglobal_load_lds_dwordx4 v0, s[2:3]\n",
               "\ts_mov_b32 m0, s4\n", "\ts_nop 0\n", "\tglobal_load_lds_dwordx4 v0, s[2:3]\n",
               "\tv_readfirstlane_b32 s3, v1\n", "\ts_mov_b32 m0, s4\n", "\ts_nop 2\n", "\tglobal_load_lds_dwordx4 v0, s[2:3]\n",
               "\tv_readfirstlane_b32 s3, v1\n", "\ts_mov_b32 m0, s4\n", "\ts_nop 3\n", "\tglobal_load_lds_dwordx4 v0, s[2:3]\n"]
    listing += ["\ts_mov_b32 s1, m0\n"]
    loads, missing = owed(listing)
    assert missing.pop() == ("s_mov_b32 s1, m0", "M0")
    assert loads == 4 and [m[0].split()[0] for m in missing] == ["s_mov_b32", "v_readfirstlane_b32"]


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_every_load_to_lds_has_its_waits(tmp_path):
    lib = tmp_path / "libsi.so"
    os.symlink(LIB_PATH, lib)
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    parts = sorted(p for p in tmp_path.iterdir() if "gfx950" in p.name)
    assert parts
    loads, missing = 0, []
    for part in parts:
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", str(part)], stdout=subprocess.PIPE, text=True) as dump:
            n, m = owed(dump.stdout)
        loads, missing = loads + n, missing + m
    assert loads > 0 and not missing, (loads, len(missing), missing[:3])
