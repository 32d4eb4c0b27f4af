"""Waits before loads into LDS, read from the built kernels: the compiler counts no wait states for loads written in assembly, so a
descriptor or an offset that a vector instruction has just written would be read before it arrives, and the load go anywhere."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2509_06980_amd as rl
from test_kernel_resources import _code_objects

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin:" + os.environ.get("PATH", ""))
FIVE = 5      # wait states between a vector instruction that writes a scalar and a memory instruction that reads it


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)", operand)
    if not m:
        return set()
    return set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}


def _too_early(listing):
    """(loads into LDS, [(load, writer)]) of a listing"""
    past, loads, bad = [], 0, []
    for line in listing.splitlines():
        text = line.split("//")[0].strip()
        if not text or text.endswith(":"):
            past = past if text.startswith("L") else []
            continue
        words = re.split(r"[\s,]+", text)
        if words[0].startswith("buffer_load") and "lds" in words:
            loads += 1
            needs, waited = set().union(*map(_scalars, words[1:])), 0
            for before in reversed(past):
                if waited >= FIVE:
                    break
                if before[0].startswith("v_read") and _scalars(before[1]) & needs:
                    bad.append((text, " ".join(before)))
                    break
                waited += int(before[1], 0) + 1 if before[0] == "s_nop" else 1
        past = past[-8:] + [words]
    return loads, bad


def test_the_reader_finds_a_load_that_comes_too_early():
    listing = "v_readfirstlane_b32 s8, v1\ns_mov_b32 m0, s3\ns_nop 0\nbuffer_load_dword v2, s[8:11], s4 offen lds\n"
    assert _too_early(listing) == (1, [("buffer_load_dword v2, s[8:11], s4 offen lds", "v_readfirstlane_b32 s8 v1")])
    assert _too_early(listing.replace("s_nop 0", "s_nop 3")) == (1, []) and _too_early(listing.replace("s8, v1", "s12, v1")) == (1, [])


@pytest.mark.skipif(not OBJDUMP, reason="no disassembler for the built kernels")
def test_descriptors_are_settled_before_loads_into_lds(tmp_path):
    if not os.path.exists(rl.LIB_PATH):
        from paper_2509_06980_amd import build
        build.build()
    loads, bad = 0, []
    for i, elf in enumerate(_code_objects(rl.LIB_PATH)):
        path = tmp_path / f"{i}.elf"
        path.write_bytes(elf)
        n, b = _too_early(subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout)
        loads, bad = loads + n, bad + b
    assert loads > 500 and not bad, bad[:5]
