"""What the compiler made of the operators' kernels, from the notes in the built library: their registers fit."""
import re
import struct

import pytest

from paper_2205_05632_amd import binding as B

msgpack = pytest.importorskip("msgpack")


def code_objects(data):
    """The GPU code objects that the library's own build put into it."""
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    at = data.find(magic)
    while at >= 0:
        (count,) = struct.unpack_from("<Q", data, at + len(magic))
        entry = at + len(magic) + 8
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + length]:
                yield data[at + offset:at + offset + size]
            entry += 24 + length
        at = data.find(magic, at + 1)


def kernels(elf):
    """name -> metadata of a code object's kernels (the note sections of a 64-bit ELF file)."""
    assert elf[:4] == b"\x7fELF"
    (table,) = struct.unpack_from("<Q", elf, 0x28)
    size, count = struct.unpack_from("<HH", elf, 0x3A)
    for i in range(count):
        _, kind, _, _, offset, length = struct.unpack_from("<IIQQQQ", elf, table + i * size)
        at, end = offset, offset + length
        while kind == 7 and at < end:
            of_name, of_desc, note = struct.unpack_from("<III", elf, at)
            desc = at + 12 + (of_name + 3) // 4 * 4
            if note == 32:    # the metadata of the kernels
                for k in msgpack.unpackb(elf[desc:desc + of_desc])["amdhsa.kernels"]:
                    yield k[".name"], k
            at = desc + (of_desc + 3) // 4 * 4


def test_registers_of_the_operators_kernels():
    """No more than eight registers of a lane are spilled (a workgroup of 1024 threads has 128 for each)."""
    found = {}
    for elf in code_objects(open(B.LIB_PATH, "rb").read()):
        found.update(kernels(elf))
    ours = {k: v for k, v in found.items() if re.search(r"k_(norm|loss|dropout)", k)}
    assert len(ours) > 100
    over = {k: v[".vgpr_spill_count"] for k, v in ours.items() if v[".vgpr_spill_count"] > 8}
    assert not over, over
