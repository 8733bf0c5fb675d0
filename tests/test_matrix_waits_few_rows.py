"""m0 in the kernels of few rows with 8-bit weights: they write it in inline assembly for their loads into LDS, as the tiles do, and the compiler does not
preserve it around those statements. Read from the disassembly of the library as it was built; needs no GPU."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from tests.test_matrix_waits import OBJDUMP, other_uses_of_m0


def as_a_tile(listing):
    """The listing with these kernels under a name that the reader looks at."""
    return listing.replace("w8_few_kernel", "gemm_tile_kernel")


def test_the_reader_sees_the_kernels_of_few_rows():
    text = "0000 <void laser::w8_few_kernel<3, 4, 4, false, false>(laser::W8Args)>:\n\ts_mov_b32 m0, s3 // 00\n\t%s // 04\n"
    assert not other_uses_of_m0(as_a_tile(text % "s_nop 0"))
    assert other_uses_of_m0(as_a_tile(text % "s_mov_b32 s4, m0")) and other_uses_of_m0(as_a_tile(text % "s_add_u32 m0, m0, s1"))


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no disassembler")
def test_m0_of_the_built_kernels(tmp_path):
    from paper_2408_05676_amd import build as b
    if not os.path.exists(b.LIB):
        b.build(verbose=False)
    shutil.copy(b.LIB, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    writes = 0
    for obj in glob.glob(str(tmp_path / "*gfx950")):
        listing = subprocess.run([OBJDUMP, "-d", "--demangle", obj], capture_output=True, text=True, check=True).stdout
        kernels = "".join(k for k in re.split(r"(?m)^(?=[0-9a-f]+ <)", listing) if "w8_few_kernel" in k.split("\n", 1)[0])
        writes += kernels.count("s_mov_b32 m0")
        assert not other_uses_of_m0(as_a_tile(kernels))
    assert writes > 100, "no loads into LDS found"
