"""Wait states in the built device code that the compiler does not look after: loads from memory
into LDS are issued from inline assembly (dma16 and its like), into which its hazard pass does
not look. The target asks for one wait state between a scalar write of M0 and a load that takes
its LDS address from there, and for five between a vector instruction's write of a scalar
register and a memory instruction that reads it."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2511_06724_amd import dn

OBJDUMP = next((c for c in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if c and os.path.exists(c)), None)


def _scalar_registers(text):
    out = set()
    for a, b, c in re.findall(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        out |= {int(c)} if c else set(range(int(a), int(b) + 1))
    return out


def _lds_loads_too_early(lines):
    """(loads seen, those with a wait state missing, each with the instruction before) of disassembled code."""
    seen, bad, code = 0, [], []
    for line in lines:
        text = line.split("//")[0].strip()
        op, _, args = text.partition(" ")
        if not args and not op.startswith("s_"):
            continue
        if "_load_lds_" in op or (op.startswith("buffer_load") and args.split()[-1] == "lds"):
            seen += 1
            states, base = 0, _scalar_registers(args)
            for prev, pargs in reversed(code[-5:]):
                dst = pargs.split(",")[0].strip()
                if (states < 1 and dst == "m0") or (states < 5 and prev.startswith("v_") and _scalar_registers(dst) & base):
                    bad.append(f"{prev} {pargs} / {text}")
                states += int(pargs, 0) + 1 if prev == "s_nop" else 1
        code.append((op, args.strip()))
    return seen, bad


def test_missing_wait_states_are_seen():
    load = "\tglobal_load_lds_dwordx4 v1, s[4:5]   // 0: 00"
    for before, ok in ((["s_mov_b32 m0, s1"], False), (["s_mov_b32 m0, s1", "s_nop 0"], True),
                       (["s_mov_b32 m0, s1", "s_add_i32 s2, s2, 1"], True),
                       (["v_readfirstlane_b32 s5, v0", "s_nop 3"], False), (["v_readfirstlane_b32 s5, v0", "s_nop 4"], True),
                       (["v_readfirstlane_b32 s6, v0", "s_nop 0"], True)):
        seen, bad = _lds_loads_too_early(before + [load])
        assert seen == 1 and (not bad) == ok, before


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_loads_into_lds_keep_their_wait_states(tmp_path):
    lib = shutil.copy(dn._LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", str(lib)], cwd=tmp_path, check=True, capture_output=True)
    seen, bad = 0, []
    for f in sorted(tmp_path.glob("lib.so.*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(f)], check=True, capture_output=True,
                              text=True).stdout
        s, b = _lds_loads_too_early(text.splitlines())
        seen, bad = seen + s, bad + b
    assert seen > 100, "the library's loads into LDS"
    assert not bad, f"{len(bad)} of {seen}: {bad[:3]}"
