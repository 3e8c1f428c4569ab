"""What the built kernels take of a compute unit, read from the library's own metadata: kernels that count on several workgroups there."""
import struct

import msgpack

from paper_2105_04779_amd.build import LIB


def _code_objects(blob):
    """The gfx950 ELF images inside the library's bundles."""
    magic = b"__CLANG_OFFLOAD_BUNDLE__"
    at = blob.find(magic)
    while at >= 0:
        count, = struct.unpack_from("<Q", blob, at + len(magic))
        p = at + len(magic) + 8
        for _ in range(count):
            offset, size, name = struct.unpack_from("<QQQ", blob, p)
            if b"gfx950" in blob[p + 24:p + 24 + name] and size:
                yield blob[at + offset:at + offset + size]
            p += 24 + name
        at = blob.find(magic, at + 1)


def _kernels(elf):
    """The kernels' metadata: the notes of type 32 (NT_AMDGPU_METADATA) are msgpack."""
    shoff, = struct.unpack_from("<Q", elf, 40)
    shentsize, shnum = struct.unpack_from("<HH", elf, 58)
    for i in range(shnum):
        kind, _, _, offset, size = struct.unpack_from("<IQQQQ", elf, shoff + i * shentsize + 4)
        if kind != 7:                                                # SHT_NOTE
            continue
        p = offset
        while p < offset + size:
            namesz, descsz, note = struct.unpack_from("<III", elf, p)
            desc = p + 12 + (namesz + 3) // 4 * 4
            if note == 32:
                yield from msgpack.unpackb(elf[desc:desc + descsz], strict_map_key=False)["amdhsa.kernels"]
            p = desc + (descsz + 3) // 4 * 4


def test_two_rows_of_logits_share_a_compute_unit():
    """Rows of up to 8 pieces a lane are taken by 16 wavefronts each.  With more than 64 registers, of 512 that a SIMD has for a lane, a compute unit holds
    one such workgroup, and nothing is under way while it computes."""
    with open(LIB, "rb") as f:
        blob = f.read()
    found = {k[".name"]: k for elf in _code_objects(blob) for k in _kernels(elf)}
    rows = {n: k for n, k in found.items() if "k_score_chunk" in n and k[".max_flat_workgroup_size"] == 1024 and "Li16E" not in n}
    assert len(rows) == 6, sorted(found)                             # three types, 4 and 8 pieces
    for name, k in rows.items():
        assert k[".vgpr_count"] <= 64 and k[".vgpr_spill_count"] == 0 and 2 * k[".group_segment_fixed_size"] <= 163840, (name, k[".vgpr_count"])
