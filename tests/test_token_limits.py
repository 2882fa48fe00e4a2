"""CPU checks of the token operators at the ends of their integers: what no launch can take is refused before anything is launched."""
import ctypes as C
import os
import subprocess

import pytest

import paper_2308_15949_amd as L
from paper_2308_15949_amd import binding as B
from paper_2308_15949_amd import build

NEAR, FAR, THIRD = 0x10000, 1 << 44, 1 << 45  # never dereferenced
vp = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        build.build(verbose=False)
    return L.load()


@pytest.mark.parametrize("M,N,out", [(1, 1 << 27, B.BF16), (16, (1 << 31) - 8, B.F32),              # 16 columns a workgroup of 512 threads
                                     (1 << 29, 8, B.BF16), ((1 << 31) - 1, 64, B.F32),              # 64 x 64 results, 512 threads
                                     ((1 << 31) - 1, (1 << 31) - 8, B.BF16)])
def test_products_of_more_threads_than_a_launch_has(lib, M, N, out):
    ld = N
    assert lib.laud_matmul_e4m3(vp(NEAR), 16, vp(NEAR), vp(FAR), 16, vp(NEAR), M, N, 16, vp(THIRD), ld, out, None, 0, None) == B.ERR_UNSUPPORTED


def test_quantisation_of_more_blocks_than_a_launch_has(lib):
    n = (1 << 31) - 8
    assert lib.laud_quantize_e4m3(vp(NEAR), n, 1, n, B.BF16, 128, vp(FAR), n, vp(THIRD), None) == B.ERR_UNSUPPORTED


def test_numbers_of_blocks(tmp_path):
    (tmp_path / "blocks.hip").write_text('#include "laud_token.h"\nextern "C" int blocks(int n) { return laud::scale_blocks(n); }\n')
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.FLAGS, "--cuda-host-only", "-shared", str(tmp_path / "blocks.hip"),
                    "-o", str(tmp_path / "blocks.so")], check=True, capture_output=True)
    blocks = C.CDLL(str(tmp_path / "blocks.so")).blocks
    for n in (0, 1, 127, 128, 129, 1 << 20, (1 << 31) - 129, (1 << 31) - 128, (1 << 31) - 127, (1 << 31) - 1):
        assert blocks(n) == -(-n // 128)
