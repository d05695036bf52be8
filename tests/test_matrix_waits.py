"""The built library's own GPU code, searched for results of matrix instructions that are read or written over too soon.

The hardware does not hold back a vector or memory instruction that takes a matrix instruction's result before it is there: the compiler
has to put wait states between them.  Where a branch joins in between it has been seen to count them along one of the ways only (a choice
by a pointer's being NULL between products and the first reader of their sums left 7 of 12 on the other), and the last registers came out
old.  This follows every way from each matrix instruction to the first reader, so that an edit or a compiler that brings it back shows."""
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2604_12841_amd as pdx
from conftest import ROOT

LIB = os.path.join(ROOT, "paper_2604_12841_amd", "libpredecoder.so")
OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"

# Wait states from a matrix instruction to a vector or memory instruction, or to another matrix one that takes its result as A or B: its passes (of
# four cycles) and four, of fp32 products two.  What is not listed counts as the longest.  (That many are in straight code of this compiler.)
WAITS = {"_4x4x4_": 6, "_16x16x32_bf16": 8, "_16x16x32_f16": 8, "_16x16x32_fp8": 8, "_16x16x64_i8": 8, "_32x32x16_bf16": 12, "_32x32x16_f16": 12,
         "_32x32x16_fp8": 12, "_32x32x32_i8": 12, "_16x16x128_f8f6f4": 12, "_16x16x4_f32": 10, "_32x32x64_f8f6f4": 20}
TAKEN = 2  # a branch that is taken: the code behind it has to be fetched, which takes longer than that


def needed(op):
    return next((n for name, n in WAITS.items() if name in op), max(WAITS.values()))


def registers(text):
    """The vector and accumulation registers that an operand list names."""
    r = set()
    for kind, lo, hi, one_kind, one in re.findall(r"\b([av])\[(\d+):(\d+)\]|\b([av])(\d+)\b", text):
        r.update((kind, n) for n in range(int(lo), int(hi) + 1)) if kind else r.add((one_kind, int(one)))
    return r


def functions(listing):
    """(name, instructions, index of each label) of a disassembly; a branch's last operand is its label."""
    name, code, labels = None, [], {}
    for line in listing.splitlines():
        m = re.match(r"^[0-9a-f]* ?<(\w+)>:", line)
        if m and re.fullmatch(r"L\d+", m.group(1)):
            labels[m.group(1)] = len(code)
        elif m:
            if name:
                yield name, code, labels
            name, code, labels = m.group(1), [], {}
        elif name and line.startswith("\t"):
            code.append(line.split("//")[0].strip())
    if name:
        yield name, code, labels


def too_soon(code, labels):
    """[(index of a matrix instruction, index of what takes its result, wait states between them)]."""
    found = []
    for i, t in enumerate(code):
        if not t.startswith("v_mfma"):
            continue
        op, operands = t.split(None, 1)
        need, result = needed(op), registers(operands.split(",")[0])
        ways, best = [(i + 1, 0)], {}
        while ways:
            j, waited = ways.pop()
            while j < len(code) and waited < need and waited < best.get(j, need):
                best[j] = waited
                op, _, operands = code[j].partition(" ")
                if op.startswith("v_mfma"):
                    parts = operands.split(",")
                    if registers(",".join(parts[1:3])) & result:
                        found.append((i, j, waited))
                        break
                    if registers(parts[0]) == result:
                        break  # a product added to it, which the hardware holds back: the search goes on from there
                elif op.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")) and registers(operands) & result:
                    found.append((i, j, waited))
                    break
                if op in ("s_endpgm", "s_setpc_b64", "s_swappc_b64"):
                    break
                waited += int(operands, 0) + 1 if op == "s_nop" else 1
                if op == "s_branch":
                    j, waited = labels[operands.split()[-1]], waited + TAKEN - 1
                    continue
                if op.startswith("s_cbranch"):
                    ways.append((labels[operands.split()[-1]], waited + TAKEN - 1))
                j += 1
    return found


def test_the_search_finds_a_short_way():
    listing = """
0000000000000000 <kernel>:
	v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], v[0:15] // 0
	s_cbranch_scc1 L0 // 1
	s_nop 15 // 2
	v_add_f32_e32 v30, v15, v31 // 3
0000000000000020 <L0>:
	s_nop 8 // 4
	v_add_f32_e32 v30, v31, v15 // 5
	s_endpgm // 6
"""
    (name, code, labels), = functions(listing)
    assert name == "kernel" and too_soon(code, labels) == [(0, 5, 11)]
    code[4] = "s_nop 9"
    assert too_soon(code, labels) == []
    code[2] = "v_mfma_f32_16x16x32_bf16 v[40:43], v[12:15], v[20:23], v[40:43]"
    assert too_soon(code, labels) == [(0, 2, 1)]


def device_code(path):
    """The gfx950 objects of a shared library: its section .hip_fatbin holds bundles, each a table of (offset, size, target) and the parts."""
    data, magic = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        n, = struct.unpack_from("<Q", data, at + len(magic))
        table = at + len(magic) + 8
        if n > 16:  # (the name alone, in a string)
            at = data.find(magic, at + 1)
            continue
        for _ in range(n):
            offset, size, length = struct.unpack_from("<3Q", data, table)
            target = data[table + 24:table + 24 + length]
            table += 24 + length
            if b"gfx950" in target and size:
                yield data[at + offset:at + offset + size]
        at = data.find(magic, at + 1)


def test_no_result_is_taken_too_soon(tmp_path):
    if not os.path.exists(LIB):
        pytest.skip("libpredecoder.so not built")
    if not shutil.which(OBJDUMP):
        pytest.skip("no llvm-objdump")
    matrix, seen = 0, set()
    for n, code in enumerate(device_code(LIB)):
        path = tmp_path / ("%d.o" % n)
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--symbolize-operands", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        for name, code, labels in functions(listing):
            found = too_soon(code, labels)
            assert not found, (name, [(code[i], code[j], waited) for i, j, waited in found[:5]])
            matrix += sum(t.startswith("v_mfma") for t in code)
            seen.add(name)
    assert matrix > 1000 and any("linear_narrow_kernel" in name for name in seen)
