"""The built whole-sequence kernels' instructions: nothing behind a branch overwrites the addend of a
matrix instruction that is still running.

A matrix instruction reads its addend's registers for some cycles after it issues.  In a straight line the
compiler keeps vector instructions and LDS reads that write them far enough away; past a branch taken right behind
matrix instructions it has been seen not to, and results of one row in four were wrong.  What decides instructions
between products is a template argument for that reason, and this looks at what came out: from every branch
back over the last wait states and on from its target over as many, no write to an addend."""

import os
import re
import subprocess

import pytest

import test_kernel_resources as T
from paper_2608_15533_amd import deltalog as D

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
KERNELS = ("forward_kernel", "both_kernel")                 # their code objects hold the others too
# Wait states.  The longest of the instructions used there takes 8 passes, and needs 7 before its addend may be
# written; the nearest write in these kernels is more than 20 away.
WINDOW = 14
REGS = re.compile(r"([va])\[(\d+):(\d+)\]|([va])(\d+)$")
WRITES = ("v_", "ds_read", "global_load", "buffer_load", "flat_load", "scratch_load")


def _regs(operand):
    m = REGS.match(operand)
    if not m:
        return frozenset()
    if m.group(1):
        return frozenset((m.group(1), i) for i in range(int(m.group(2)), int(m.group(3)) + 1))
    return frozenset([(m.group(4), int(m.group(5)))])


def _parse(listing):
    """[(address, opcode, operands, branch target or None)] of a disassembly."""
    symbols, out = {}, []
    for line in listing.splitlines():
        if line.startswith("0"):
            m = re.match(r"([0-9a-f]+) <([^>]+)>:", line)
            if m:
                symbols[m.group(2)] = int(m.group(1), 16)
            continue
        if not line.startswith("\t"):
            continue
        text, _, note = line.partition("//")
        words = text.split(None, 1)
        m = re.match(r"\s*([0-9A-F]+):[^<]*(?:<([^>+]+)(?:\+0x([0-9a-f]+))?>)?", note)
        if m is None:                                      # padding
            continue
        target = None
        if words[0].startswith(("s_cbranch", "s_branch")):
            target = (m.group(2), int(m.group(3) or "0", 16))
        operands = [x.strip() for x in words[1].split(",")] if len(words) > 1 else []
        out.append((int(m.group(1), 16), words[0], operands, target))
    return [(a, op, ops, None if t is None else symbols[t[0]] + t[1]) for a, op, ops, t in out]


def _states(op, operands):
    return int(operands[0]) + 1 if op == "s_nop" else 1


def _written(op, operands):
    if not op.startswith(WRITES) or op.startswith(("v_cmp", "v_mfma")) or not operands:
        return frozenset()
    return _regs(operands[0])


def overwritten(code, window=WINDOW):
    """(branch, matrix instruction, write) addresses where a write to an addend's registers lies within the window."""
    at = {a: i for i, (a, _, _, _) in enumerate(code)}
    hits = []
    for i, (address, _, _, target) in enumerate(code):
        if target is None:
            continue
        running, back = [], 0
        for j in range(i - 1, -1, -1):
            a, op, operands, t = code[j]
            if t is not None or op.startswith(("s_barrier", "s_endpgm")):
                break
            back += _states(op, operands)
            if back > window:
                break
            if op.startswith("v_mfma"):
                running.append((back, a, _regs(operands[3]) | _regs(operands[0])))
        if not running:
            continue
        on, k = 0, at[target]
        while k < len(code) and on < window:
            a, op, operands, _ = code[k]
            if op.startswith(("s_waitcnt", "s_barrier")):
                break
            on += _states(op, operands)
            w = _written(op, operands)
            hits += [(address, m, a) for d, m, r in running if w & r and d + on <= window]
            k += 1
    return hits


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_no_addend_is_overwritten_behind_a_branch(tmp_path):
    with open(D.LIB_PATH, "rb") as f:
        blob = f.read()
    seen, bad = 0, {}
    for n, elf in enumerate(T._code_objects(blob)):
        if not any(k in name for name, _ in T._descriptors(elf) for k in KERNELS):
            continue
        path = tmp_path / f"{n}.elf"
        path.write_bytes(elf)
        code = _parse(subprocess.run([OBJDUMP, "-d", str(path)], capture_output=True, text=True,
                                     check=True).stdout)
        seen += sum(op.startswith("v_mfma") for _, op, _, _ in code)
        bad[n] = [tuple(map(hex, h)) for h in overwritten(code)]
    assert seen > 10000                                    # the parser found the kernels
    assert not any(bad.values()), bad


LISTING = """
0000000000001000 <k>:
	v_mfma_f32_16x16x4_f32 v[8:11], v0, v1, v[4:7]             // 000000001000: D3C50008 0412030D
	s_cbranch_scc1 2                                           // 000000001008: BF850002 <k+0x14>
	s_nop 0                                                    // 00000000100C: BF800000
	s_nop 0                                                    // 000000001010: BF800000
	{gap}// 000000001014: BF800000
	{write}// 000000001018: 7E0C0300
	s_endpgm                                                   // 00000000101C: BF810000
"""


@pytest.mark.parametrize("gap,write,hit", [
    ("s_nop 0 ", "v_mov_b32_e32 v6, v0 ", True), ("s_nop 0 ", "v_mov_b32_e32 v12, v0 ", False),
    ("s_nop 15 ", "v_mov_b32_e32 v6, v0 ", False), ("s_waitcnt lgkmcnt(0) ", "v_mov_b32_e32 v6, v0 ", False),
    ("s_nop 1 ", "ds_read_b128 v[2:5], v20 ", True)])
def test_the_search_finds_what_it_looks_for(gap, write, hit):
    assert bool(overwritten(_parse(LISTING.format(gap=gap, write=write)))) == hit
