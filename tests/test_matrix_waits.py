"""Results of the matrix cores in the machine code of this library: an instruction that reads them, or writes their registers, has to come a number of wait
states behind the product, or it reads what was there before.  The compiler sees to that within a block and mostly across them; where two ways of different
length join it has not always.  Here every way through every kernel is followed."""
import os
import re
import struct
import subprocess

import pytest

from test_kernel_resources import LIB

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
# passes of 4 cycles: 4 for tiles of 16 x 16, 8 for 32 x 32, and 4 more wait states until other instructions than products may read or write the result
WAITS = {"16x16": 8, "32x32": 12}
REGISTERS = re.compile(r"\b([va])\[(\d+):(\d+)\]|\b([va])(\d+)\b")
NO_RESULT = ("global_store", "buffer_store", "flat_store", "scratch_store", "ds_write", "global_atomic", "buffer_atomic", "ds_add", "ds_min", "ds_max", "ds_or",
             "v_cmp", "v_readfirstlane", "v_readlane", "global_load_lds")


def code_objects():
    """The library's own, one to a source file."""
    data, at, magic = open(LIB, "rb").read(), 0, b"__CLANG_OFFLOAD_BUNDLE__"
    while (at := data.find(magic, at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, p)
            if size and b"gfx950" in data[p + 24:p + 24 + length]:
                yield data[at + offset:at + offset + size]
            p += 24 + length
        at += len(magic)


def registers(text):
    found = set()
    for kind, first, last, one, number in REGISTERS.findall(text):
        found |= {(kind, i) for i in range(int(first), int(last) + 1)} if kind else {(one, int(number))}
    return found


def matrix(op):
    return op.startswith(("v_mfma", "v_smfma"))


def operands(op, text):
    """(registers written, registers read, the sum that a product adds to)."""
    parts = re.split(r",(?![^\[]*\])", text)
    if matrix(op):
        return registers(parts[0]), registers(",".join(parts[1:3])), registers(parts[3]) if len(parts) > 3 else set()
    if not op.startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_")):
        return set(), set(), set()
    if op.startswith(NO_RESULT) or text.rstrip().endswith(" lds"):
        return set(), registers(text), set()
    both = op.startswith(("v_fmac", "v_dot2c", "v_dot4c", "v_pk_fmac", "v_swap")) or "swap" in op
    return registers(parts[0]), registers(text if both else ",".join(parts[1:])), set()


def too_early(code):
    """code: [(op, operands' text, target's index or None)] of one kernel: [(product, reader, wait states)]."""
    parsed, found = {}, []
    for start, (name, text, _) in enumerate(code):
        if not matrix(name):
            continue
        need = next(n for shape, n in WAITS.items() if shape in name)
        ways, seen = [(start + 1, 0, frozenset(operands(name, text)[0]))], {}
        while ways:
            at, states, live = ways.pop()
            while at < len(code) and states < need and live:
                if seen.get((at, live), need) <= states:
                    break
                seen[at, live] = states
                op, text, target = code[at]
                if at not in parsed:
                    parsed[at] = operands(op, text)
                written, read, added = parsed[at]
                if live & (read if matrix(op) else read | written):
                    found.append(("%s %s" % (name, code[start][1]), "%s %s" % (op, text), states))
                live = live - read - written - added
                states += 1 + (int(text, 0) if op == "s_nop" else 0)
                if op == "s_endpgm":
                    break
                if op.startswith("s_cbranch"):
                    ways.append((target, states, live))
                at = target if op == "s_branch" else at + 1
    return found


def kernels_of(path):
    """Kernels of a code object: (name, code)."""
    line = re.compile(r"^\t(\S+)\s*(.*?)\s*// ([0-9A-F]+):[^<]*(?:<.*\+0x([0-9a-f]+)>|<.*>)?$")
    name, code = None, []

    def done():
        index = {address: i for i, (_, _, address, _) in enumerate(code)}
        return name, [(op, text, index.get(offset + code[0][2]) if offset is not None else None) for op, text, _, offset in code]

    dump = subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", path], stdout=subprocess.PIPE, text=True)
    for row in dump.stdout:
        if row.startswith("0") and row.rstrip().endswith(">:"):
            if code:
                yield done()
            name, code = row[row.index("<") + 1:-3], []
        elif row.startswith("\t") and row.strip() != "...":
            op, text, address, offset = line.match(row.rstrip()).groups()
            branch = op.startswith(("s_cbranch", "s_branch"))
            code.append((op, text, int(address, 16), (int(offset, 16) if offset else 0) if branch else None))
    if code:
        yield done()
    assert dump.wait() == 0


def test_a_reader_that_comes_too_early_is_found():
    product, reader, nop = ("v_mfma_f32_16x16x32_f16", "v[0:3], v[8:11], v[12:15], v[0:3]", None), ("v_mul_f32_e32", "v9, v4, v1", None), ("s_nop", "6", None)
    end = ("s_endpgm", "", None)
    assert too_early([product, nop, reader, end]) and not too_early([product, nop, nop, reader, end])
    assert too_early([product, ("s_nop", "7", None), reader, end]) == []
    # the shorter of two ways to the reader: over the branch
    ways = [product, ("s_cbranch_scc1", "4", 4), nop, nop, reader, end]
    assert [w[2] for w in too_early(ways)] == [1]
    # a product that adds to the result needs no wait, one that multiplies with it does
    assert not too_early([product, product, nop, nop, reader, end])
    assert too_early([product, ("v_mfma_f32_16x16x32_f16", "v[20:23], v[0:3], v[12:15], 0", None), nop, nop, end])


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_results_of_the_matrix_cores_are_waited_for(tmp_path):
    if not os.path.exists(LIB):
        import __graft_entry__
        __graft_entry__.build()
    products, early = 0, []
    for i, elf in enumerate(code_objects()):
        path = tmp_path / ("%d.co" % i)
        path.write_bytes(elf)
        for name, code in kernels_of(str(path)):
            n = sum(matrix(op) for op, _, _ in code)
            if n:
                products += n
                early += [(name,) + e for e in too_early(code)]
        path.unlink()
    assert products > 10000
    assert not early, early[:5]
