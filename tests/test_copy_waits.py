"""The copies from memory into LDS in the built library, instruction by instruction.

They are written out as assembly, which the compiler does not look into, so that the waits that gfx950 leaves to the program are the source's own
to bring: one wait state between a scalar write of m0 and the copy that reads it, and five between a vector instruction that writes a
scalar register and a memory instruction that reads it.  An instruction is one wait state, s_nop n is n + 1."""
import os
import re
import struct
import subprocess

import pytest

import paper_2602_17206_amd as pkg

OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
BUNDLE = b"__CLANG_OFFLOAD_BUNDLE__"


def code_objects(library):
    """The gfx950 code objects of every source in the library"""
    with open(library, "rb") as f:
        data = f.read()
    at = data.find(BUNDLE)
    while at >= 0:
        entry = at + len(BUNDLE) + 8
        for _ in range(struct.unpack_from("<Q", data, entry - 8)[0]):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if size and b"gfx950" in data[entry + 24:entry + 24 + length]:
                yield data[at + offset:at + offset + size]
            entry += 24 + length
        at = data.find(BUNDLE, at + 1)


def scalars(operand):
    """The scalar registers that an operand names"""
    many = re.fullmatch(r"s\[(\d+):(\d+)\]", operand)
    if many:
        return {"s%d" % r for r in range(int(many[1]), int(many[2]) + 1)}
    return {operand} if re.fullmatch(r"s\d+|m0", operand) else set()


def short_waits(listing):
    """(copies, those that come too early): each with its kernel"""
    copies, early, kernel, before = 0, [], None, []
    for line in listing:
        name = re.match(r"[0-9a-f]+ <(.*)>:", line)
        if name:
            kernel, before = name[1], []
            continue
        words = line.split("//")[0].split(None, 1)
        if not words:
            continue
        op, operands = words[0], [x.strip() for x in words[1].split(",")] if len(words) > 1 else []
        if op.startswith(("buffer_load", "global_load")) and "lds" in " ".join([op] + operands).split():
            copies += 1
            reads = set().union(*(scalars(x) for each in operands for x in each.split()))
            states = 0
            for was, to in reversed(before):
                if states >= 5:
                    break
                # (a carry or a comparison's result is the first or the second operand)
                writes = set().union(*(scalars(x) for x in to[:2 if was.startswith("v_") else 1]))
                if was.startswith("v_") and writes & reads:
                    early.append((kernel, was, states))
                if was.startswith("s_") and not was.startswith("s_nop") and "m0" in writes and states < 1:
                    early.append((kernel, was, states))
                states += int(to[0], 0) + 1 if was == "s_nop" else 1
        before = before[-8:] + [(op, operands)]
    return copies, early


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_copies_into_lds_wait_for_their_scalar_registers(tmp_path):
    pkg.load_library()
    copies = 0
    for n, code in enumerate(code_objects(pkg.library_path())):
        path = tmp_path / ("%d.elf" % n)
        path.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        found, early = short_waits(listing.splitlines())
        assert not early, (len(early), found, early[:3])
        copies += found
    assert copies > 0


def test_what_counts_as_too_early():
    listing = ["0 <kernel>:", "v_readfirstlane_b32 s6, v1", "s_mov_b32 m0, s2", "%s", "buffer_load_dwordx4 v55, s[4:7], 0 offen lds"]
    for nop, early in (("s_nop 3", 0), ("s_nop 2", 1), ("s_nop 0", 1), ("", 2)):
        assert [len(x) if isinstance(x, list) else x for x in short_waits([line.replace("%s", nop) for line in listing])] == [1, early], nop
    listing[1] = "v_readfirstlane_b32 s8, v1"
    assert short_waits([line.replace("%s", "s_nop 0") for line in listing]) == (1, [])
