"""Matrix instructions' results in the built library are not read, nor their registers written, before they are there.

The hardware does not hold back an ordinary instruction that touches the result of a matrix instruction under way: the compiler has to place it
far enough behind.  Across a short branch it once did not, and the first elements of a result were stale.  So every matrix instruction
in the device code of libob.so is followed along every path, and whatever touches its result too early fails.

Wait states are counted as the compiler counts them: one an instruction, s_nop n + 1.  What is needed behind an instruction of `passes` passes of four clocks:
passes + 4 for 16-bit types, passes + 2 for fp32, before a vector, memory or LDS instruction touches the result or another matrix
instruction has it as a factor; passes - 1 for 16-bit types before a vector instruction overwrites the addend.  (A matrix instruction that
adds to a result is held back by the hardware.)"""
import re
import shutil
import struct
import subprocess
from pathlib import Path

import pytest

from paper_1705_07860_amd import binding

OBJDUMP = shutil.which("llvm-objdump", path="/opt/rocm/llvm/bin") or shutil.which("llvm-objdump")
PASSES = {"16x16x4": 8, "16x16x16": 4, "16x16x32": 4, "4x4x": 2, "32x32x2": 16, "32x32x8": 8, "32x32x16": 8}


def passes(name):
    return PASSES[next(k for k in sorted(PASSES, key=len, reverse=True) if k in name)]


def needed(name):
    return passes(name) + (2 if re.search(r"(x2|x4)_?f32$", name) else 4)


def registers(text):
    """The vector registers that an operand names."""
    got = set()
    for kind, lo, hi, one in re.findall(r"(?<![\w.])([va])(?:\[(\d+):(\d+)\]|(\d+))(?!\w)", text):
        got |= {(kind, i) for i in (range(int(lo), int(hi) + 1) if lo else (int(one),))}
    return got


def kernels(text):
    """{kernel: [(address, instruction, target of its branch)]} from a disassembly."""
    got, code, start = {}, None, 0
    for line in text.splitlines():
        m = re.match(r"^([0-9a-f]+) <(.+)>:$", line)
        if m:
            start, code = int(m[1], 16), got.setdefault(m[2], [])
            continue
        m = re.match(r"^\t(.+?)\s*// ([0-9A-F]+):(.*)$", line)
        if m and code is not None:
            to = re.search(r"<.+\+0x([0-9a-f]+)>", m[3])
            code.append((int(m[2], 16), m[1].strip(), start + int(to[1], 16) if to else None))
    return got


def too_early(code):
    """(matrix instructions, [(one, what touches its result, wait states between)]) of one kernel."""
    at = {address: i for i, (address, _, _) in enumerate(code)}
    total, found = 0, []
    for i, (_, text, _) in enumerate(code):
        if not text.startswith("v_mfma"):
            continue
        name, rest = text.split(None, 1)
        result, need = registers(rest.split(",")[0]), needed(name)
        total += 1
        addend = registers(re.split(r",\s*(?![^\[]*\])", rest)[3]) if not re.search(r"(x2|x4)_?f32$", name) else set()
        held = passes(name) - 1
        seen, todo = {}, [(i + 1, 0)]
        while todo:
            j, waits = todo.pop()
            if waits >= need or j >= len(code) or seen.get(j, need) <= waits:
                continue
            seen[j] = waits
            _, other, target = code[j]
            op, _, args = other.partition(" ")
            if op == "s_endpgm":
                continue
            if op.startswith(("s_branch", "s_cbranch")):
                todo.append((at[target], waits + 1))
                if op == "s_branch":
                    continue
            elif op.startswith("v_mfma"):
                # result, factor, factor, addend
                parts = re.split(r",\s*(?![^\[]*\])", args)
                if (registers(parts[1]) | registers(parts[2])) & result:
                    found.append((text, other, waits))
                    continue
                if (registers(parts[0]) | registers(parts[3])) & result:    # held back until it is there; who comes next counts from that one
                    continue
            elif registers(args) & result or (waits < held and op.startswith("v_") and registers(args.split(",")[0]) & addend):
                found.append((text, other, waits))
                continue
            todo.append((j + 1, waits + 1 + (int(args, 0) if op == "s_nop" else 0)))
    return total, found


def device_code(library):
    data, at = library.read_bytes(), 0
    while (at := data.find(b"__CLANG_OFFLOAD_BUNDLE__", at)) >= 0:
        count, place = struct.unpack_from("<Q", data, at + 24)[0], at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, place)
            if size and b"gfx950" in data[place + 24:place + 24 + length]:
                yield data[at + offset:at + offset + size]
            place += 24 + length
        at += 24


def test_the_walk_finds_what_is_planted():
    mfma = "v_mfma_f32_16x16x32_bf16 v[4:7], v[8:11], v[12:15], v[4:7]"

    def code(*lines):
        return [(4 * i, text, target) for i, (text, target) in enumerate(x if isinstance(x, tuple) else (x, None) for x in lines)]
    assert too_early(code(mfma, "s_nop 7", "v_mul_f32_e32 v1, v2, v4")) == (1, [])
    assert too_early(code(mfma, "s_nop 6", "v_mul_f32_e32 v1, v2, v4"))[1]
    assert too_early(code(mfma, "s_nop 6", "ds_write_b64 v1, v[6:7] offset:16"))[1]
    assert not too_early(code(mfma, "s_nop 0", "ds_write_b64 v1, v[16:17]", "s_nop 7"))[1]
    assert too_early(code(mfma, "v_mfma_f32_16x16x32_bf16 v[20:23], v[4:7], v[12:15], v[20:23]"))[1]
    assert not too_early(code(mfma, mfma, "s_nop 7", "v_mov_b32_e32 v1, v4"))[1]
    # only the jump is short
    assert too_early(code(mfma, ("s_cbranch_scc1 6", 12), "s_nop 7", "v_mov_b32_e32 v1, v4"))[1]
    assert not too_early(code(mfma, ("s_cbranch_scc1 6", 16), "s_nop 7", "v_mov_b32_e32 v1, v4", "s_nop 7"))[1]
    assert too_early(code("v_mov_b32_e32 v1, v4", "s_nop 2", mfma, ("s_branch 0", 0)))[1]
    assert needed("v_mfma_f32_16x16x4_f32") == 10 and needed("v_mfma_f32_16x16x32_f16") == 8


@pytest.mark.skipif(not OBJDUMP, reason="no llvm-objdump here")
def test_no_matrix_result_is_touched_too_early(tmp_path):
    if not binding.LIB_PATH.exists():
        from paper_1705_07860_amd import build
        build.build()
    total = 0
    for n, code in enumerate(device_code(Path(binding.LIB_PATH))):
        elf = tmp_path / f"{n}.elf"
        elf.write_bytes(code)
        text = subprocess.run([OBJDUMP, "-d", str(elf)], capture_output=True, text=True, check=True).stdout
        for kernel, lines in kernels(text).items():
            count, found = too_early(lines)
            total += count
            assert not found, (kernel, found[:3])
    assert total > 1000                                   # the walk saw them
