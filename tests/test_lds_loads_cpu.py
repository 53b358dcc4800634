"""The wait states that gfx950 wants ahead of a load from memory to LDS, in the code that was built.  Compilers see to them between
instructions of their own and not within or around an inline assembly block, and the loads of the prompt kernels' tiles are such blocks:
  a scalar write of m0 (the address in LDS), one other instruction, then the load that goes by it
  a vector instruction's write of the scalar base address, five wait states, then the load that reads it."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2407_02328_amd import LIB_PATH

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin") or shutil.which("llvm-objdump")
WRITES_SCALARS = re.compile(r"^v_(readfirstlane|readlane|cmp)\w*$")


def scalars(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if m is None:
        return {"vcc"} if operand.startswith("vcc") else set()
    return set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}


def hazards(lines):
    """Loads to LDS that follow too soon on what they need, and how many loads there are; lines: (mnemonic, operands)."""
    found, loads = [], 0
    for i, (name, args) in enumerate(lines):
        if not ("_load_lds_" in name or (name.startswith("buffer_load") and args[-1:] == ["lds"])):
            continue
        loads += 1
        base = set().union(*(scalars(a) for a in args))
        waited = 0                       # wait states between line j and the load
        for j in range(i - 1, -1, -1):
            other, what = lines[j]
            if waited < 1 and what[:1] == ["m0"] and other.startswith("s_"):
                found.append((i, "m0"))
            if WRITES_SCALARS.match(other) and what and base & scalars(what[0]):
                found.append((i, "base"))
            waited += int(what[0], 0) + 1 if other == "s_nop" else 1
            if waited >= 5:
                break
    return found, loads


def parsed(text):
    lines = []
    for line in text.splitlines():
        line = line.split("//")[0].strip()
        if not line or line.endswith(":") or not re.match(r"[a-z]", line) or "file format" in line:
            continue
        name, _, rest = line.partition(" ")
        lines.append((name, re.split(r",\s*|\s+", rest.strip()) if rest.strip() else []))
    return lines


@pytest.mark.parametrize("text,want", [
    ("s_mov_b32 m0, s3\nglobal_load_lds_dwordx4 v4, s[0:1]", ["m0"]),
    ("s_mov_b32 m0, s3\ns_nop 0\nglobal_load_lds_dwordx4 v4, s[0:1]", []),
    ("v_readfirstlane_b32 s1, v0\ns_mov_b32 m0, s3\ns_nop 0\nglobal_load_lds_dwordx4 v4, s[0:1]", ["base"]),
    ("v_readfirstlane_b32 s2, v0\ns_mov_b32 m0, s3\ns_nop 0\nglobal_load_lds_dwordx4 v4, s[0:1]", []),
    ("v_readfirstlane_b32 s1, v0\ns_nop 2\ns_mov_b32 m0, s3\ns_nop 0\nglobal_load_lds_dwordx4 v4, s[0:1]", []),
])
def test_the_search_finds_them(text, want):
    assert [what for _, what in hazards(parsed(text))[0]] == want


@pytest.mark.skipif(OBJDUMP is None, reason="no llvm-objdump")
def test_loads_to_lds_wait_for_their_addresses(tmp_path):
    if not os.path.exists(LIB_PATH):
        from paper_2407_02328_amd.build import build_library
        build_library()
    library = shutil.copy(LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", str(library)], check=True, capture_output=True, timeout=60, cwd=tmp_path)
    total = 0
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" not in name:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], check=True, capture_output=True, timeout=300, text=True, cwd=tmp_path).stdout
        lines = parsed(text)
        found, loads = hazards(lines)
        total += loads
        assert not found, f"{name}: {len(found)} of {loads} loads, the first: {lines[found[0][0] - 2:found[0][0] + 1]}, {found[0][1]}"
    assert total > 0, "no load to LDS in the library"
