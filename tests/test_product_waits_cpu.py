"""Matrix products' results in the built library: on every path through a kernel, enough wait states lie between a product and the first instruction of another
kind that touches its result (or a product that takes it as a factor). The hardware does not wait by itself, and the compiler has left the waits out where a
result is moved right behind a short branch: a kernel of one wave a SIMD, whose products go to accumulation registers, then gives other numbers from
run to run. Read from the disassembly of the library that is there, without a GPU."""
from __future__ import annotations

import functools
import os
import re
import shutil
import struct
import subprocess

import pytest

import paper_2609_24875_amd as pkg

OBJDUMP = next((p for p in ("/opt/rocm/llvm/bin/llvm-objdump", shutil.which("llvm-objdump")) if p and os.path.exists(p)), None)
PASSES = {"4x4x4": 2, "16x16x16": 4, "16x16x32": 4, "32x32x8": 8, "32x32x16": 8}


def _wait_states(passes):
    """That the compiler itself keeps on gfx950 where it sees one path only: 5, 8 and 12 for products of 2, 4 and 8 passes of four cycles."""
    return passes + 3 + (passes > 2)


@functools.lru_cache(maxsize=None)
def _registers(operands):
    """The vector and accumulation registers that operands name."""
    found = set()
    for kind, lo, hi, one in re.findall(r"\b([va])(?:\[(\d+):(\d+)\]|(\d+))(?![\w\[])", operands):
        found |= {(kind, i) for i in range(int(lo or one), int(hi or one) + 1)}
    return frozenset(found)


@functools.lru_cache(maxsize=None)
def _operands(text):
    return re.split(r",\s*(?![^\[]*\])", text)


def _functions(listing):
    """(name, [(instruction, operands, place of a branch's target or None)]) of each function of a disassembly."""
    name, start, ins, at = None, 0, [], {}

    def done():
        return name, [(op, rest, at.get(to) if to is not None else None) for op, rest, to in ins]
    for line in listing.splitlines():
        m = re.match(r"^([0-9a-f]+) <(\S+)>:$", line)
        if m:
            if name is not None:
                yield done()
            start, name, ins, at = int(m.group(1), 16), m.group(2), [], {}
            continue
        text, _, rest = line.partition("//")
        text = text.strip()
        if name is None or not rest or not text:
            continue
        op, _, operands = text.partition(" ")
        at[int(rest.split(":")[0], 16)] = len(ins)
        to = re.search(r"<\S+?(?:\+0x([0-9a-f]+))?>\s*$", rest) if op.startswith(("s_branch", "s_cbranch")) else None
        ins.append((op, operands.strip(), start + int(to.group(1) or "0", 16) if to else None))
    if name is not None:
        yield done()


def _too_early(ins):
    """(products, [(product, instruction, wait states between, wait states needed)])"""
    products, found = 0, []
    for i, (op, rest, _) in enumerate(ins):
        if "mfma" not in op:
            continue
        products += 1
        result = _registers(_operands(rest)[0])
        need = _wait_states(PASSES[re.search(r"_(\d+x\d+x\d+)", op).group(1)])
        best, todo = {}, [(i + 1, 0)]
        while todo:
            j, waited = todo.pop()
            if j is None or j >= len(ins) or waited >= need or best.get(j, need) <= waited:
                continue
            best[j] = waited
            op2, rest2, to = ins[j]
            if "mfma" in op2:
                d, a, b, c = _operands(rest2)[:4]
                # (a sum that goes on from the whole result is forwarded; products write in order)
                if (_registers(a) | _registers(b)) & result or (_registers(c) & result and _registers(c) != result):
                    found.append((f"{op} {rest}", f"{op2} {rest2}", waited, need))
                if _registers(d) >= result:
                    continue
            elif op2.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")) and _registers(rest2) & result:
                found.append((f"{op} {rest}", f"{op2} {rest2}", waited, need))
                continue
            waited += int(rest2, 0) + 1 if op2 == "s_nop" else 1
            if op2 == "s_branch":
                todo.append((to, waited))
            elif op2 != "s_endpgm":
                todo += [(j + 1, waited)] + ([(to, waited)] if to is not None else [])
    return products, found


def _listing(*lines):
    return "0000000000000100 <k>:\n" + "".join(f"\t{line}    // {0x100 + 4 * i:012X}: 00000000{to}\n"
                                                for i, (line, to) in enumerate((x, "") if isinstance(x, str) else x for x in lines))


PRODUCT = "v_mfma_f32_32x32x16_f16 a[0:15], v[2:5], v[78:81], a[0:15]"


@pytest.mark.parametrize("lines,early", [
    ([PRODUCT, "s_nop 11", "v_accvgpr_read_b32 v17, a15", "s_endpgm"], None),
    ([PRODUCT, "s_nop 10", "v_accvgpr_read_b32 v17, a15", "s_endpgm"], 11),
    # a branch around what would have been long enough
    ([PRODUCT, ("s_cbranch_vccnz 12", " <k+0x38>"), *["v_add_f32_e32 v2, v2, v3"] * 12, "v_accvgpr_read_b32 v17, a15", "s_endpgm"], 1),
    ([PRODUCT, ("s_cbranch_vccnz 12", " <k+0x38>"), *["v_add_f32_e32 v2, v2, v3"] * 12, "s_nop 11", "v_accvgpr_read_b32 v17, a15", "s_endpgm"], None),
    # around a loop's end
    (["v_mov_b32_e32 v9, a3", PRODUCT, ("s_branch 65533", " <k>")], 1),
    (["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "s_nop 6", "ds_write_b128 v20, v[0:3]", "s_endpgm"], 7),
    (["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "s_nop 7", "ds_write_b128 v20, v[0:3]", "s_endpgm"], None),
    (["v_mfma_f32_4x4x4_16b_f16 v[0:3], v[8:9], v[12:13], 0", "s_nop 3", "v_mov_b32_e32 v2, 0", "s_endpgm"], 4),
    # sums that go on, factors, parts of a sum
    ([PRODUCT, PRODUCT, "s_nop 11", "v_accvgpr_read_b32 v17, a15", "s_endpgm"], None),
    (["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "v_mfma_f32_16x16x32_f16 v[4:7], v[0:3], v[12:15], 0", "s_endpgm"], 0),
    (["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "v_mfma_f32_16x16x32_f16 v[2:5], v[8:11], v[12:15], v[2:5]", "s_endpgm"], 0),
    (["v_mfma_f32_16x16x32_f16 v[0:3], v[8:11], v[12:15], 0", "v_mfma_f32_16x16x32_f16 v[2:5], v[8:11], v[12:15], v[0:3]", "s_nop 7",
      "v_add_f32_e32 v2, v2, v0", "s_endpgm"], None)])
def test_what_counts_as_too_early(lines, early):
    (name, ins), = _functions(_listing(*lines))
    products, found = _too_early(ins)
    assert name == "k" and products == sum("mfma" in str(x) for x in lines)
    assert [f[2] for f in found] == ([] if early is None else [early])


def _code_objects(path):
    """The device code of every source in the library: bundles of (offset, size, target)."""
    data, magic = open(path, "rb").read(), b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        p = at + 32
        for _ in range(count):
            off, size, n = struct.unpack_from("<QQQ", data, p)
            if b"gfx950" in data[p + 24:p + 24 + n] and size:
                yield data[at + off:at + off + size]
            p += 24 + n
        at = data.find(magic, at + 24)


@pytest.mark.skipif(OBJDUMP is None or not os.path.exists(pkg.LIB_PATH), reason="libsph.so not built, or no disassembler")
def test_no_result_is_touched_too_early(tmp_path):
    kernels = products = 0
    early = {}
    for i, code in enumerate(_code_objects(pkg.LIB_PATH)):
        f = tmp_path / f"{i}.co"
        f.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(f)], capture_output=True, text=True, check=True).stdout
        for name, ins in _functions("\n".join(f for f in listing.split("\n\n") if "v_mfma" in f)):
            n, found = _too_early(ins)
            kernels, products = kernels + (n > 0), products + n
            if found:
                early[name] = found[:3]
    assert kernels > 100 and products > 10000            # (that something was read at all)
    assert not early
