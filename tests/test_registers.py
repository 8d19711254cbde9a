"""What the built library's code objects say of its kernels' registers.

A vector register that is spilled to scratch is stored by the lanes that are active at the store. hipcc has placed such a store at the head of a block where a
divergent loop's lanes meet again, in front of the instruction that makes them active: the lanes that had left the loop kept nothing, and what they had summed up to
there was lost. A kernel without spilled vector registers has no such store."""
import struct

import pytest

msgpack = pytest.importorskip("msgpack")

BUNDLE, SHT_NOTE, NT_AMDGPU_METADATA = b"__CLANG_OFFLOAD_BUNDLE__", 7, 32


def code_objects(library):
    """The gfx950 code objects that the compiler bundled into the library."""
    at = library.find(BUNDLE)
    while at >= 0:
        n, = struct.unpack_from("<Q", library, at + 24)
        entry = at + 32
        for _ in range(n):
            offset, size, length = struct.unpack_from("<QQQ", library, entry)
            if b"gfx950" in library[entry + 24:entry + 24 + length]:
                yield library[at + offset:at + offset + size]
            entry += 24 + length
        at = library.find(BUNDLE, at + 24)


def kernels(elf):
    """The metadata of a code object's kernels, from its note sections."""
    sections, = struct.unpack_from("<Q", elf, 40)
    size, n = struct.unpack_from("<HH", elf, 58)
    for s in range(n):
        kind, = struct.unpack_from("<I", elf, sections + s * size + 4)
        at, length = struct.unpack_from("<QQ", elf, sections + s * size + 24)
        end = at + length if kind == SHT_NOTE else at
        while at < end:
            name, words, note = struct.unpack_from("<III", elf, at)
            at += 12 + (name + 3) // 4 * 4
            if note == NT_AMDGPU_METADATA:
                yield from msgpack.unpackb(elf[at:at + words])["amdhsa.kernels"]
            at += (words + 3) // 4 * 4


@pytest.fixture(scope="module")
def spilled():
    from paper_2301_07482_amd import binding

    with open(binding.LIB_PATH, "rb") as f:
        found = {k[".name"]: k[".vgpr_spill_count"] for elf in code_objects(f.read()) for k in kernels(elf)}
    assert found
    return found


@pytest.mark.parametrize("part", ["group_norm", "distill", "grouped", "gated", ""])
def test_no_kernel_spills_vector_registers(spilled, part):
    of_part = {name: n for name, n in spilled.items() if part in name}
    assert of_part
    # 16 steps of load_linear_kernel's contraction: six registers of W's columns and of an address, which do not change in its loop. They are stored in front of it, in
    # straight code, by the lanes that run it.
    assert {name: n for name, n in of_part.items() if n and "load_linear_kernelILi16E" not in name} == {}
    assert all(n <= 6 for n in of_part.values())
