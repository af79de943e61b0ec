"""The built device code of the experts' products, whose loads to LDS are written out in assembly, disassembled and
read: the compiler puts no wait states inside an assembly block or between one and the code around it.  No GPU is needed."""
import os
import re
import struct
import subprocess

import pytest

from paper_1705_01598_amd import binding as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
WAIT = 5        # states between a vector instruction that writes a scalar register and a vector memory one that reads it


def _code_objects():
    """gfx950 code objects of the library that hold an experts' product."""
    B.lib()
    data = open(B.LIB_PATH, "rb").read()
    at = data.find(MAGIC)
    while at >= 0:
        entry = at + len(MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, at + len(MAGIC))[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            target = data[entry + 24:entry + 24 + length]
            entry += 24 + length
            code = data[at + offset:at + offset + size]
            if target.endswith(b"gfx950") and b"expert_product_kernel" in code:
                yield code
        at = data.find(MAGIC, at + 1)


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if m:
        return set(range(int(m[1]), int(m[2]) + 1))
    return {int(operand[1:])} if re.fullmatch(r"s\d+", operand) else {operand} if operand in ("m0", "vcc") else set()


def _too_early(instructions, k):
    """The vector instruction less than WAIT states in front of load k that writes a scalar which it reads, or None."""
    need = {"m0"}.union(*(_scalars(o) for o in instructions[k][1:]))
    passed = 0
    for op, *operands in reversed(instructions[max(0, k - WAIT):k]):
        written = operands[:1] if op.startswith(("v_readfirstlane", "v_readlane", "v_cmp")) else \
            operands[1:2] if "_co_" in op or op.startswith(("v_mad_u64", "v_mad_i64", "v_div_scale")) else []
        if any(_scalars(o) & need for o in written):
            return op, operands
        passed += int(operands[0], 0) + 1 if op == "s_nop" else 1
        if passed >= WAIT:
            return None
    return None


def test_the_reader_finds_what_it_looks_for():
    load = ["buffer_load_dwordx4", "v4", "s[4:7]", "s23", "offen", "lds"]
    write = ["v_readfirstlane_b32", "s4", "v2"]
    for between, early in (([], True), ([["s_mov_b32", "m0", "s9"], ["s_nop", "0"]], True), ([["s_nop", "3"]], True), ([["s_nop", "4"]], False),
                           ([["s_mov_b32", "m0", "s9"], ["s_nop", "3"]], False)):
        code = [write, *between, load]
        assert bool(_too_early(code, len(code) - 1)) == early
    assert _too_early([["v_mad_u64_u32", "v[2:3]", "s[6:7]", "s2", "v4", "v[2:3]"], load], 1)
    assert not _too_early([["v_readfirstlane_b32", "s8", "v2"], load], 1) and not _too_early([["s_add_u32", "s4", "s4", "s5"], load], 1)


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_loads_to_lds_keep_their_distance_from_the_scalars_they_read(tmp_path):
    loads = objects = 0
    for code in _code_objects():
        objects += 1
        path = tmp_path / "code.elf"
        path.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        kernel, instructions = "", []
        for line in text.splitlines():
            if line.startswith("\t"):
                instructions.append(re.split(r"[,\s]+", line.split("//")[0].strip()))
                if instructions[-1][0].startswith("buffer_load") and instructions[-1][-1] == "lds":
                    loads += 1
                    assert not _too_early(instructions, len(instructions) - 1), (kernel, instructions[-WAIT - 1:])
            elif line.endswith(">:"):
                kernel, instructions = line.split("<")[1], []
    assert objects == 3 and loads > 100
