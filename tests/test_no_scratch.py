"""The product kernels of the built library use no scratch memory.

Their K loops count the loads in flight themselves (vmcnt); spilled registers' loads and stores
between those would be counted too.  The int8 kernels of 256x256 tiles keep 4 registers in scratch
memory, written before a tile's first load and read before or after its K loop: no more than that.
The sizes stand in the code objects' metadata, one code object per source."""
import os
import re
import shutil
import struct
import subprocess

import pytest

from paper_2205_01848_amd import binding as B
from paper_2205_01848_amd.build import ARCH

READELF = shutil.which("llvm-readelf") or "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"
PRODUCTS = re.compile(r"ffn_gemm|ffn_few_rows")
I8_TILES = re.compile(r"ffn_gemm16_kernelILi[678]E")


def code_objects(lib):
    at = lib.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", lib, at + len(MAGIC))
        entry = at + len(MAGIC) + 8
        for _ in range(count):
            offset, size, n = struct.unpack_from("<3Q", lib, entry)
            name = lib[entry + 24:entry + 24 + n].decode()
            entry += 24 + n
            if name.endswith(ARCH):
                yield lib[at + offset:at + offset + size]
        at = lib.find(MAGIC, at + 1)


def scratch_sizes(code, path):
    """{kernel: bytes of scratch memory a lane} of a code object."""
    path.write_bytes(code)
    text = subprocess.run([READELF, "--notes", str(path)], capture_output=True, text=True, check=True).stdout
    names = re.findall(r"^\s+\.name:\s+'?(_Z\w+)'?$", text, re.M)
    sizes = re.findall(r"\.private_segment_fixed_size:\s+(\d+)", text)
    assert len(names) == len(sizes)
    return dict(zip(names, map(int, sizes)))


@pytest.mark.skipif(not os.path.exists(READELF), reason="llvm-readelf is not installed")
def test_products_use_no_scratch_memory(tmp_path):
    with open(B.LIB_PATH, "rb") as f:
        lib = f.read()
    sizes = {}
    for i, code in enumerate(code_objects(lib)):
        sizes.update(scratch_sizes(code, tmp_path / f"{i}.o"))
    products = {k: v for k, v in sizes.items() if PRODUCTS.search(k)}
    vocab = [k for k in products if re.search(r"_kernelILi1[345]E", k)]
    assert len(products) > 100 and len(vocab) >= 10
    tiles = {k: v for k, v in products.items() if I8_TILES.search(k)}
    assert len(tiles) == 3 and all(v <= 20 for v in tiles.values()), tiles
    assert not {k: v for k, v in products.items() if v and k not in tiles}
