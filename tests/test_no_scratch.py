"""Kernels over the cache keep everything in registers: what the built library says of their scratch memory."""
import struct

import msgpack

from paper_2602_11688_amd.build import LIB

AMDGPU, METADATA = 224, 32                            # ELF machine, note type


def _kernels():
    """Name and bytes of scratch memory a lane, of every kernel of the library."""
    data = open(LIB, "rb").read()
    at = data.find(b"\x7fELF", 4)
    while at >= 0:
        if struct.unpack_from("<H", data, at + 18)[0] == AMDGPU:
            sections, = struct.unpack_from("<Q", data, at + 40)
            size, count = struct.unpack_from("<HH", data, at + 58)
            for i in range(count):
                kind, = struct.unpack_from("<I", data, at + sections + i * size + 4)
                offset, length = struct.unpack_from("<QQ", data, at + sections + i * size + 24)
                if kind == 7:                         # notes
                    note, end = at + offset, at + offset + length
                    while note < end:
                        name, desc, type = struct.unpack_from("<III", data, note)
                        begin = note + 12 + (name + 3) // 4 * 4
                        if type == METADATA:
                            for kernel in msgpack.unpackb(data[begin:begin + desc])["amdhsa.kernels"]:
                                yield kernel[".name"], kernel[".private_segment_fixed_size"]
                        note = begin + (desc + 3) // 4 * 4
        at = data.find(b"\x7fELF", at + 4)


def test_attention_and_appends():
    found = {name: scratch for name, scratch in _kernels() if any(part in name for part in ("attend_", "join_prompt", "append_kernel", "kv_"))}
    assert len(found) > 100
    assert {name: scratch for name, scratch in found.items() if scratch} == {}
