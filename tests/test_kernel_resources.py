"""What the compiler gave the kernels of the built library, from the metadata beside their code (no GPU)."""
import struct

import msgpack

from .helpers import ensure_built

MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def kernels(path):
    """The metadata record of every kernel in the library's gfx950 code objects."""
    data = open(path, "rb").read()
    found = []
    at = data.find(MAGIC)
    while at >= 0:
        (count,) = struct.unpack_from("<Q", data, at + len(MAGIC))
        entry = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, n = struct.unpack_from("<QQQ", data, entry)
            name = data[entry + 24:entry + 24 + n]
            entry += 24 + n
            if b"gfx950" in name and size:
                found += notes(data[at + offset:at + offset + size])
        at = data.find(MAGIC, at + 1)
    return found


def notes(elf):
    """amdhsa.kernels of one code object."""
    (start,) = struct.unpack_from("<Q", elf, 32)          # program headers
    size, count = struct.unpack_from("<HH", elf, 54)
    for i in range(count):
        kind, _, offset, _, _, length = struct.unpack_from("<IIQQQQ", elf, start + i * size)
        end = offset + length
        while kind == 4 and offset + 12 <= end:            # notes: name "AMDGPU", type 32: the metadata
            name, desc, what = struct.unpack_from("<III", elf, offset)
            body = offset + 12 + (name + 3) // 4 * 4
            if what == 32 and elf[offset + 12:offset + 18] == b"AMDGPU":
                return msgpack.unpackb(elf[body:body + desc])["amdhsa.kernels"]
            offset = body + (desc + 3) // 4 * 4
    return []


def test_medium_batch_kernels_use_no_scratch():
    """Their ring lies in registers: a spilled register is stored and loaded in every step (up to 14 % of the kernel)."""
    found = {k[".name"]: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for k in kernels(ensure_built().LIB_PATH) if "midm_kernel" in k[".name"]}
    assert len(found) == 11   # nibbles in groups of 128 and bytes with one to four blocks of 16 rows, groups of 64 with up to three
    assert set(found.values()) == {(0, 0)}, found


def test_serving_kernels_use_no_scratch():
    """A row of a norm, a tile's results and its operands lie in registers.  The exception is the norm's gradient beyond 8192 columns: 1024 threads with 128
    registers each hold two or four pieces of the row, of the next one and of the weight's sums."""
    names = ("rmsnorm", "kv_append", "attend_", "join_", "adapters_")
    found = {k[".name"]: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for k in kernels(ensure_built().LIB_PATH) if any(n in k[".name"] for n in names)}
    assert len(found) == 47, sorted(found)   # 14 and 6 + 1 of the norm, 4 of the writer, 4 + 4 and 2 + 2 of the attention, 4 + 4 + 2 of the adapters
    wide = {n for n in found if "rmsnorm_back_kernelILi1024ELi2E" in n or "rmsnorm_back_kernelILi1024ELi4E" in n}
    assert len(wide) == 2
    assert {n: v for n, v in found.items() if n not in wide and v != (0, 0)} == {}


def test_kernels_of_the_policys_ends_use_no_scratch():
    """Sums, fragments and a row of logits lie in registers."""
    names = ("embed_", "w16a16_", "sample_kernel")
    found = {k[".name"]: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for k in kernels(ensure_built().LIB_PATH) if any(n in k[".name"] for n in names)}
    assert len(found) == 34, sorted(found)   # lookup, 6 of the sort, parts, 2 of the rows; 15 products and 3 beside them; 6 of the sampling
    assert {n: v for n, v in found.items() if v != (0, 0)} == {}
