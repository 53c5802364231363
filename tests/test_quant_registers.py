"""What the compiler made of the kernels in 8-bit integers, by the metadata of the built library: no kernel of theirs keeps values of a
row or a tile in memory of its own (runs without a GPU)."""
import re
import struct
import subprocess
from pathlib import Path

import pytest

import paper_2605_11186_amd as cats

READELF = Path("/opt/rocm/llvm/bin/llvm-readelf")
pytestmark = pytest.mark.skipif(not READELF.exists(), reason="ROCm's readelf is not there")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def device_objects():
    """The gfx950 code objects of the library, one for each source file."""
    blob = cats.library_path().read_bytes()
    at = blob.find(MAGIC)
    while at >= 0:
        count, = struct.unpack_from("<Q", blob, at + len(MAGIC))
        entry = at + len(MAGIC) + 8
        for _ in range(count if count < 8 else 0):
            offset, size, length = struct.unpack_from("<QQQ", blob, entry)
            target = blob[entry + 24:entry + 24 + length]
            if target.endswith(b"gfx950") and size:
                yield blob[at + offset:at + offset + size]
            entry += 24 + length
        at = blob.find(MAGIC, at + 1)


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Name of each kernel in 8-bit integers -> bytes of memory of its own that a thread has."""
    found, path = {}, tmp_path_factory.mktemp("objects") / "object"
    for obj in device_objects():
        path.write_bytes(obj)
        notes = subprocess.run([str(READELF), "--notes", str(path)], check=True, capture_output=True, text=True).stdout
        for name, size in re.findall(r"\.name:\s+(\S+)\n(?:(?!\s+\.name:).*\n)*?\s+\.private_segment_fixed_size:\s+(\d+)", notes):
            if "cats_quant" in name:
                found[name] = int(size)
    return found


def test_no_kernel_spills(kernels):
    assert sum("quantize_rows" in n for n in kernels) > 100 and sum("linear_split" in n for n in kernels) > 20
    assert {n: size for n, size in kernels.items() if size} == {}


def test_norms_of_several_pieces_are_of_rows_that_layers_have(kernels):
    """Rows of hidden columns, at most 8192: 64 to 512 threads with 1, 2 or 3 pieces of 8 values each, aligned or not."""
    cut = sorted(re.search(r"pieces_tELi(\d+)ELi(\d+)", n).groups() for n in kernels if "pieces_t" in n)
    assert cut == sorted([("64", "1"), ("256", "1"), ("256", "2"), ("256", "3"), ("512", "2")] * 2)
