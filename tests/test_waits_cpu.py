"""Waits that assembly written by hand has to bring itself, looked up in the built code.

The compiler keeps gfx950's distances between dependent instructions, but it does not look into inline assembly.  A load
straight to LDS takes its place there from M0 and needs one instruction or wait state between it and the scalar write
of M0; a scalar register that a vector instruction wrote needs five before a memory instruction reads it.
"""
from __future__ import annotations

import os
import re
import struct
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_33184_amd", "libspecstream.so")
OBJCOPY = "/opt/rocm/llvm/bin/llvm-objcopy"
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _numbers(operand):
    """Numbers of the scalar registers that an operand names."""
    m = re.fullmatch(r"s(\d+)", operand)
    if m:
        return {int(m[1])}
    m = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    return set(range(int(m[1]), int(m[2]) + 1)) if m else set()


def _states(op, operands):
    return int(operands[0], 0) + 1 if op == "s_nop" else 1


def faults(listing):
    """Of a listing (one instruction a line): loads straight to LDS that follow what they depend on too closely."""
    lines = []
    for line in listing.splitlines():
        m = re.match(r"\s+([a-z]\w+)\s*(.*?)\s*(//.*)?$", line)
        if m:
            lines.append((m[1], [x.strip() for x in re.split(r",(?![^\[]*\])", m[2])]))
    found, loads = [], 0
    for i, (op, operands) in enumerate(lines):
        direct = "load_lds" in op or op.startswith("buffer_load") and operands[-1].split()[-1] == "lds"
        if not direct:
            continue
        loads += 1
        reads = set().union(*(_numbers(x.split()[0]) for x in operands if x))
        apart = 0
        for before, args in lines[i - 1::-1] if i else []:
            if apart >= 5:
                break
            if args and args[0] == "m0" and apart < 1:
                found.append((op, operands, before, args))
            if before.startswith("v_") and args and _numbers(args[0]) & reads:
                found.append((op, operands, before, args))
            apart += _states(before, args)
    return loads, found


def test_faults_are_seen():
    """The rule itself, on listings written here."""
    bad = "\ts_mov_b32 m0, s9\n\tglobal_load_lds_dwordx4 v1, s[6:7]\n"
    good = "\ts_mov_b32 m0, s9\n\ts_nop 0\n\tglobal_load_lds_dwordx4 v1, s[6:7]\n"
    assert faults(bad)[0] == 1 and len(faults(bad)[1]) == 1
    assert faults(good) == (1, [])
    near = "\tv_readfirstlane_b32 s7, v2\n\ts_mov_b32 m0, s9\n\ts_nop 2\n\tglobal_load_lds_dwordx4 v1, s[6:7]\n"
    assert len(faults(near)[1]) == 1 and faults(near.replace("s_nop 2", "s_nop 3")) == (1, [])
    assert len(faults("\ts_mov_b32 m0, s9\n\tbuffer_load_dword v1, s[4:7], 0 offen lds\n")[1]) == 1


def test_loads_straight_to_lds_wait_for_what_they_read(tmp_path):
    if not (os.path.exists(LIB) and os.path.exists(OBJCOPY) and os.path.exists(OBJDUMP)):
        pytest.skip("needs the built library and the ROCm binary tools")
    section = tmp_path / "fatbin"
    subprocess.run([OBJCOPY, f"--dump-section=.hip_fatbin={section}", LIB, str(tmp_path / "out.so")], check=True)
    data = section.read_bytes()
    loads = 0
    for m in re.finditer(MAGIC, data):
        at = m.start()
        n, = struct.unpack_from("<Q", data, at + len(MAGIC))
        p = at + len(MAGIC) + 8
        for _ in range(n):
            off, size, idlen = struct.unpack_from("<QQQ", data, p)
            target = data[p + 24:p + 24 + idlen].decode()
            p += 24 + idlen
            if "gfx950" not in target:
                continue
            elf = tmp_path / f"code{at}"
            elf.write_bytes(data[at + off:at + off + size])
            listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(elf)], check=True, capture_output=True, text=True).stdout
            some, found = faults(listing)
            loads += some
            assert not found, found[:3]
    assert loads > 0, "no load straight to LDS in the library"
