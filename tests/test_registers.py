"""Registers of the kernels that are bound by how many wavefronts run at a time, read from what the built library says of its own kernels.

A SIMD has 512 registers for a lane, dealt out in eights: four wavefronts run at a time with up to 128 each."""
import os
import re
import struct

import pytest

import paper_2103_13744_amd as kn

msgpack = pytest.importorskip("msgpack")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def notes(elf):
    """The metadata of a gfx950 code object: a note of type 32, in msgpack."""
    at, size, count = struct.unpack_from("<Q", elf, 40)[0], *struct.unpack_from("<HH", elf, 58)
    for i in range(count):
        kind, start, length = struct.unpack_from("<I", elf, at + size * i + 4)[0], *struct.unpack_from("<QQ", elf, at + size * i + 24)
        pos = start
        while kind == 7 and pos < start + length:  # SHT_NOTE
            name, desc, type_ = struct.unpack_from("<III", elf, pos)
            data = pos + 12 + (name + 3) // 4 * 4
            if type_ == 32 and elf[pos + 12:pos + 18] == b"AMDGPU":
                yield msgpack.unpackb(elf[data:data + desc], strict_map_key=False)
            pos = data + (desc + 3) // 4 * 4


def kernels():
    """{name: what the code object says} of all kernels of the library: its code objects are bundles, one per source."""
    kn.load_library()
    with open(os.path.join(os.path.dirname(kn.__file__), "libkilonerf_hip.so"), "rb") as f:
        lib = f.read()
    found = {}
    for m in re.finditer(MAGIC, lib):
        pos = m.end()
        (entries,) = struct.unpack_from("<Q", lib, pos)
        pos += 8
        for _ in range(entries):
            offset, size, length = struct.unpack_from("<QQQ", lib, pos)
            target = lib[pos + 24:pos + 24 + length]
            pos += 24 + length
            if b"gfx950" in target and size:
                for note in notes(lib[m.start() + offset:m.start() + offset + size]):
                    found.update({k[".name"]: k for k in note["amdhsa.kernels"]})
    return found


@pytest.fixture(scope="module")
def built():
    found = kernels()
    assert len(found) > 100, len(found)
    return found


def wavefronts(kernel):
    return min(8, 512 // max(8, -(-kernel[".vgpr_count"] // 8) * 8))


# (the first template argument behind the type: whether a mask is read from what kn_save_f8 left, which costs registers)
CASES = [(4, r"k_product_smallI%sLb0ELb1ELi2ELi4ELb0EE" % t) for t in ("DF16_", "DF16b")]  # the layers of a grid of small networks: 524,288 rows of 4,096 networks 64 x 64, forward
CASES += [(4, r"k_product_rowsI%sLb0ELb%dELb1ELi128ELi128ELi2ELi4ELi2EE" % (t, c)) for t in ("DF16_", "DF16b") for c in (0, 1)]  # tiles that two workgroups of eight share a CU for


@pytest.mark.parametrize("least,name", CASES)
def test_as_many_wavefronts_run_as_a_kernel_was_laid_out_for(built, least, name):
    hits = [k for n, k in built.items() if re.search(name, n)]
    assert len(hits) == 1, name
    assert wavefronts(hits[0]) >= least and hits[0][".private_segment_fixed_size"] == 0, hits[0][".vgpr_count"]
