"""Waits before loads into LDS along every path through the built kernels: a scalar that a vector instruction writes has to be five wait states old when a load written in assembly
takes it, also where the two stand on both ends of a loop or in blocks that branch to each other; and the products' kernels keep no scalars in vector registers."""
import os
import re
import subprocess

import pytest

import paper_2509_06980_amd as rl
from test_kernel_resources import _code_objects, _kernels
from test_load_waits import FIVE, OBJDUMP


def _scalars(operand):
    m = re.fullmatch(r"s\[(\d+):(\d+)\]|s(\d+)|(vcc(?:_lo|_hi)?)", operand)
    if not m:
        return set()
    if m[4]:
        return {"vcc": {106, 107}, "vcc_lo": {106}, "vcc_hi": {107}}[m[4]]
    return set(range(int(m[1]), int(m[2]) + 1)) if m[1] else {int(m[3])}


def _too_early(function):
    """(loads into LDS, [(load, writer)]) of one function's listing: instructions with their addresses behind //."""
    code, place = [], {}
    for line in function.splitlines():
        m = re.match(r"\s+(\S.*?)\s*// ([0-9A-F]+):", line)
        if m:
            place[int(m[2], 16)] = len(code)
            code.append((int(m[2], 16), re.split(r"[\s,]+", m[1])))
    before = [[] for _ in code]
    for i, (address, words) in enumerate(code):
        if re.match(r"s_c?branch", words[0]):
            distance = int(words[1])
            before[place[address + 4 + 4 * (distance - 65536 if distance >= 32768 else distance)]].append(i)
        assert not words[0].startswith(("s_setpc", "s_swappc", "s_call")), words      # paths that this does not follow
        if words[0] not in ("s_branch", "s_endpgm") and i + 1 < len(code):
            before[i + 1].append(i)
    loads, bad = 0, []
    for i, (_, words) in enumerate(code):
        if not (words[0].startswith("buffer_load") and "lds" in words):
            continue
        loads += 1
        needs, seen, todo = set().union(*map(_scalars, words[1:])), set(), [(p, 0) for p in before[i]]
        while todo:
            at, waited = todo.pop()
            if waited >= FIVE or (at, waited) in seen:
                continue
            seen.add((at, waited))
            other = code[at][1]
            if other[0].startswith("v_") and any(_scalars(w) & needs for w in other[1:3 if "_co_" in other[0] or "div_scale" in other[0] else 2]):
                bad.append((" ".join(words), " ".join(other)))
                continue
            waited += int(other[1], 0) + 1 if other[0] == "s_nop" else 1
            todo += [(p, waited) for p in before[at]]
    return loads, bad


def _listing(*instructions):
    return "0 <kernel>:\n" + "".join(f"\t{text}  // {4 * i:012X}: 00000000\n" for i, text in enumerate(instructions))


LOAD = "buffer_load_dwordx4 v1, s[8:11], s4 offen lds"


def test_the_reader_follows_loops_and_branches():
    # the writer at the end of a loop's body, its load at the beginning: in the order of the listing nothing is before it
    loop = ["s_mov_b32 s0, 0", "s_mov_b32 m0, s3", "s_nop 0", LOAD, "s_nop 7", "v_readlane_b32 s4, v9, 0", "s_cbranch_scc1 65530", "s_endpgm"]
    assert _too_early(_listing(*loop)) == (1, [(LOAD.replace(",", ""), "v_readlane_b32 s4 v9 0")])
    assert _too_early(_listing(*loop[:2], "s_nop 2", *loop[3:])) == (1, [])
    assert _too_early(_listing(*loop[:5], "v_readlane_b32 s5, v9, 0", *loop[6:])) == (1, [])
    # and in a block that jumps to the load, over a wait that only the other way comes by
    jump = ["s_cbranch_scc1 2", "s_nop 4", "s_branch 3", "v_cmp_eq_u32_e64 s[8:9], v1, v2", "s_branch 1", "s_endpgm", "s_nop 0", LOAD, "s_endpgm"]
    assert _too_early(_listing(*jump)) == (1, [(LOAD.replace(",", ""), "v_cmp_eq_u32_e64 s[8:9] v1 v2")])
    assert _too_early(_listing(*jump[:3], "v_mov_b32_e32 v3, s8", *jump[4:])) == (1, [])


@pytest.mark.skipif(not OBJDUMP, reason="no disassembler for the built kernels")
def test_scalars_are_settled_on_every_path_to_a_load_into_lds(tmp_path):
    if not os.path.exists(rl.LIB_PATH):
        from paper_2509_06980_amd import build
        build.build()
    loads, bad = 0, []
    for i, elf in enumerate(_code_objects(rl.LIB_PATH)):
        path = tmp_path / f"{i}.elf"
        path.write_bytes(elf)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", path], capture_output=True, text=True, check=True).stdout
        for function in re.split(r"\n(?=[0-9a-f]+ <)", listing):
            if re.search(r"\blds\b", function):
                n, b = _too_early(function)
                loads, bad = loads + n, bad + [(function[:150], *x) for x in b]
    assert loads > 2000 and not bad, bad[:5]


def test_products_keep_no_scalars_in_vector_registers():
    if not os.path.exists(rl.LIB_PATH):
        from paper_2509_06980_amd import build
        build.build()
    products = [k for k in _kernels(rl.LIB_PATH)["product", ()] if "product_kernel" in k[".name"]]
    assert len(products) > 30
    assert not [(k[".name"], k[".sgpr_spill_count"]) for k in products if k[".sgpr_spill_count"]]
