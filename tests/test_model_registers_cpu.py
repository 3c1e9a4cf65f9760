"""Whether the model operators' kernels fit beside a resident worker, from the metadata of the code objects in the built library."""
import struct

import pytest

from paper_2604_17861_amd import build as B

msgpack = pytest.importorskip("msgpack")


def kernels():
    """The metadata of every kernel, by its (mangled) name."""
    data, found = open(B.LIB, "rb").read(), {}
    magic, at = b"__CLANG_OFFLOAD_BUNDLE__", 0
    while (at := data.find(magic, at)) >= 0:
        (n,), entry = struct.unpack_from("<Q", data, at + len(magic)), at + len(magic) + 8
        for _ in range(n if n < 16 else 0):                  # (the name itself is in the library's code too)
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            target = data[entry + 24:entry + 24 + length]
            entry += 24 + length
            if not target.endswith(b"gfx950"):
                continue
            code = data[at + offset:at + offset + size]
            name = code.find(b"AMDGPU\0\0")                  # a note: sizes of name and content, type 32, name, content
            while name >= 0:
                sizes = struct.unpack_from("<III", code, name - 12)
                if sizes[0] == 7 and sizes[2] == 32:
                    for k in msgpack.unpackb(code[name + 8:name + 8 + sizes[1]])["amdhsa.kernels"]:
                        found[k[".name"]] = k
                name = code.find(b"AMDGPU\0\0", name + 1)
        at += len(magic)
    return found


def test_every_kernel_has_room_beside_the_default_worker():
    """Three workgroups of the worker leave a quarter of the registers of every SIMD, and what they leave of 160 KB."""
    all_kernels = kernels()
    model = {n: k for n, k in all_kernels.items() if "gpuos_model_kernel" in n}
    (worker,) = [k for n, k in all_kernels.items() if "gpuos_worker_kernel" in n]
    assert len(model) == 27 and worker[".vgpr_count"] <= 128 and worker[".max_flat_workgroup_size"] == 256
    for name, k in model.items():
        waves = -(-k[".max_flat_workgroup_size"] // 256)      # of a block, on each of four SIMDs
        registers = -(-k[".vgpr_count"] // 8) * 8      # (accumulation registers among them)
        assert waves * registers <= 512 - 3 * 128, (name, registers, waves)
        assert k[".group_segment_fixed_size"] <= 160 * 1024 - 3 * worker[".group_segment_fixed_size"], name
        assert k[".private_segment_fixed_size"] == 0, name
