"""How many blocks of 256 threads an SM holds of the append without rotation: as its registers allow (65,536 an SM, handed out to a warp by 256), which a second launch bound of one block once cost it."""
import os
import re
import subprocess

import pytest

from paper_2012_01114_b200 import build


@pytest.fixture(scope="module")
def registers(tmp_path_factory):
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    out = subprocess.run([nvcc, "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xptxas=-v", "-cubin", "-o", str(tmp_path_factory.mktemp("append") / "append.cubin"),
                          os.path.join(build.CSRC, "psa_cache_append.cu")], capture_output=True, text=True, check=True).stderr
    found = re.findall(r"Compiling entry function '\S*cache_append_kernelILi(\d+)ELb(\d)ELb(\d)E.*?Used (\d+) registers", out, re.S)
    return {(int(d), int(f16), int(rot)): int(n) for d, f16, rot, n in found}


@pytest.mark.parametrize("d,blocks", [(32, 6), (64, 4), (96, 3), (128, 3), (256, 2)])
def test_blocks_an_sm(registers, d, blocks):
    for f16 in (0, 1):
        warp = -(-registers[d, f16, 0] * 32 // 256) * 256
        assert 65536 // warp // 8 >= blocks
