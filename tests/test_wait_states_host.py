"""Machine code of the built library: a vector register's last write is two wait states or more before an instruction that
reads it in other lanes.  The compiler looks after that for instructions of its own, not for those of inline assembly."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2602_06935_amd import binding

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


def registers(operand):
    m = re.match(r"v\[(\d+):(\d+)\]$", operand) or re.match(r"v(\d+)$", operand)
    return set(range(int(m[1]), int(m[m.lastindex]) + 1)) if m else set()


def uses_too_early(lines):
    """Of a listing: how many instructions read lanes of a register, and those that come too early."""
    before, uses, early = [], 0, []
    for line in lines:
        line = line.split("//")[0].strip()
        if not line or line.endswith(":") or line.startswith((".", ";", "#")):
            continue
        op, _, rest = line.partition(" ")
        operands = [o.strip().split(" ")[0] for o in rest.split(",")]
        if op.endswith("_dpp"):
            uses += 1
            states = 0
            for was, its in reversed(before):
                if states >= 2:
                    break
                if was.startswith("v_") and not was.startswith("v_cmp") and registers(its[0]) & registers(operands[1]):
                    early.append((was, its, op, operands))
                    break
                states += int(its[0], 0) + 1 if was == "s_nop" else 1
        before = before[-3:] + [(op, operands)]
    return uses, early


def test_what_is_looked_for():
    use = "v_fmac_f32_dpp v0, v1, v2 row_newbcast:3 row_mask:0xf bank_mask:0xf"
    assert uses_too_early(["v_mov_b32_e32 v1, v9", use])[1]
    assert uses_too_early(["v_mov_b32_e32 v1, v9", "s_nop 0", use])[1]
    assert uses_too_early(["v_pk_mul_f32 v[0:1], v[2:3], v[4:5]", "v_mov_b32_e32 v7, v9", use])[1]
    assert uses_too_early(["v_mov_b32_e32 v1, v9", "s_nop 1", use]) == (1, [])
    assert uses_too_early(["v_mov_b32_e32 v1, v9", "v_mov_b32_e32 v7, v9", "v_mov_b32_e32 v8, v9", use]) == (1, [])
    assert uses_too_early(["v_mov_b32_e32 v2, v9", use]) == (1, [])


def test_the_built_library(tmp_path):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no disassembler")
    binding.load_library()
    shutil.copy(binding.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    uses = 0
    for name in sorted(os.listdir(tmp_path)):
        if "gfx950" not in name or b"chunk_" not in (tmp_path / name).read_bytes():
            continue
        out = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", name], cwd=tmp_path, check=True, capture_output=True, text=True)
        found, early = uses_too_early(out.stdout.splitlines())
        uses += found
        assert early == [], name
    assert uses > 0
