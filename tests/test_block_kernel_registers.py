"""Registers that the kernels of the norm, the 8-bit product and dropout spill, from the metadata the compiler wrote into the built library: the widest rows and
the 256 x 256 tile use all that a wave has, everything else fits."""
import os
import re
import struct
import subprocess

import pytest

from paper_2603_21090_amd import binding

READELF = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath("/opt/rocm/bin/hipcc"))), "llvm", "bin", "llvm-readelf")
KERNEL = re.compile(r"N4stgn(?:4norm|6dense8|4drop)\d+(\w+?_kernel)I(.*)EEv")
TYPE = {"f": "f32", "DF16b": "bf16", "DF16_": "f16", "a": "i8"}


@pytest.fixture(scope="module")
def spills(tmp_path_factory):
    """(kernel, type, its numbers) -> (spilled vector registers, bytes of scratch memory a lane)"""
    if not os.path.exists(binding.LIB_PATH):
        from paper_2603_21090_amd import build
        build.build_library()
    blob = open(binding.LIB_PATH, "rb").read()
    magic, out, at = b"__CLANG_OFFLOAD_BUNDLE__", {}, 0
    while (at := blob.find(magic, at)) >= 0:
        p = at + len(magic) + 8
        for _ in range(struct.unpack_from("<Q", blob, p - 8)[0]):
            off, size, n = struct.unpack_from("<QQQ", blob, p)
            triple = blob[p + 24:p + 24 + n]
            p += 24 + n
            if b"gfx950" not in triple or size == 0:
                continue
            obj = tmp_path_factory.mktemp("objects") / "code.o"
            obj.write_bytes(blob[at + off:at + off + size])
            text = subprocess.run([READELF, "--notes", str(obj)], capture_output=True, text=True, check=True).stdout
            for block in re.split(r"\n  - ", text):            # (a kernel's entry)
                if (name := re.search(r"\.name:\s+(\S+)", block)) and (m := KERNEL.search(name[1])):
                    dt = next(v for k, v in TYPE.items() if m[2].startswith(k))
                    numbers = tuple(map(int, re.findall(r"L(?:i|NS0_4KindE)(\d+)", m[2])))
                    out[(m[1], dt) + numbers] = tuple(int(re.search(rf"\.{field}:\s+(\d+)", block)[1]) for field in ("vgpr_spill_count", "private_segment_fixed_size"))
        at += len(magic)
    return out


def most(kernel, dt, *numbers):
    if kernel == "rows_kernel" and numbers[:2] == (512, 4):   # fp32 rows of 4,097 to 8,192, held to 128 registers for two workgroups a CU
        return (12, 24, 0)[numbers[2]]
    if kernel == "rows_kernel" and numbers[:2] == (1024, 4):  # rows of 8,193 to 16,384 in fp32 and twice that in 16 bits; a wave has 128 registers there
        return (4, 14, 0)[numbers[2]]
    if kernel == "grad_kernel" and numbers == (512, 8 if dt == "f32" else 4):        # 32 numbers a lane
        return 8
    if kernel == "turns_kernel":                              # 128 of its 256 registers are sums
        return 2
    return 0


def test_what_is_spilled(spills):
    assert {"rows_kernel", "long_rows_kernel", "grad_kernel", "columns_kernel", "fragments_kernel", "product_kernel", "direct_kernel", "turns_kernel",
            "dropout_kernel"} <= {k[0] for k in spills}
    assert {k[1] for k in spills if k[0] == "rows_kernel"} == {"f32", "bf16", "f16"}
    for key, (spilled, scratch) in spills.items():
        assert spilled <= most(*key), (key, spilled)
        assert spilled or not scratch, (key, scratch)
