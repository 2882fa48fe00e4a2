"""CPU checks of the token operators: a result over anything else that the call reads or writes is refused before a launch; arrays that
share no byte are not, wherever they stand."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2308_15949_amd as L
from paper_2308_15949_amd import binding as B
from paper_2308_15949_amd import build

vp = C.c_void_p
AT = {n: (i + 1) << 32 for i, n in enumerate(("x", "y", "keep", "gate", "out", "z", "zs", "post_w", "post_b", "pre_w", "pre_b", "a", "sa", "b",
                                              "sb", "q", "s", "router", "up", "down", "s_up", "s_down", "experts", "weights", "ws"))}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        build.build(verbose=False)
    return L.load()


def norm(lib, **over):  # 3 rows of 256 channels, 512 apart, in 8 bits with two scales a row
    at = {**AT, **over}
    p = B.NormBlock(256, B.BF16, B.NORM_LAYER, 1e-5, at["post_w"], at["post_b"], at["pre_w"], at["pre_b"], 1.0, 1.0)
    return lib.laud_norm_residual(C.byref(p), 3, vp(at["x"]), 512, vp(at["y"]), 512, vp(at["keep"]), vp(at["gate"]), 2, vp(at["out"]), 512,
                                  vp(at["z"]), 512, B.E4M3, vp(at["zs"]), None)


ROW, SCALES, VECTOR = 512, 24, 1024  # bytes: a row of x, y and out; the scales; a vector of 256


@pytest.mark.parametrize("over", [
    dict(zs=AT["x"]), dict(zs=AT["y"] + 1024 + ROW - 4), dict(zs=AT["out"] + 2048 - SCALES + 4), dict(zs=AT["z"] + 512 + 252),
    dict(out=AT["post_w"]), dict(z=AT["post_b"] + VECTOR - 16), dict(out=AT["pre_w"] - 16), dict(z=AT["pre_b"] - 16),
    dict(out=AT["gate"] + 2 * VECTOR - 16), dict(z=AT["gate"] + VECTOR), dict(keep=AT["out"] + 1024), dict(keep=AT["z"] - 2), dict(zs=AT["gate"]),
    dict(zs=AT["keep"]), dict(zs=AT["pre_w"] + VECTOR - 4)])
def test_norm(lib, over):
    assert norm(lib, **over) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("s", [AT["x"], AT["x"] + 2 * 1024 + 508, AT["q"], AT["q"] + 512 + 252, AT["x"] - 4, AT["q"] - 4])
def test_quantisation(lib, block_rows, s):
    assert lib.laud_quantize_e4m3(vp(AT["x"]), 512, 3, 256, B.BF16, block_rows, vp(AT["q"]), 512, vp(s), None) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(sa=AT["out"] + 64 * 4 - 4), dict(sa=AT["out"] - 20), dict(sb=AT["out"] + 2 * 1024), dict(sb=AT["out"] - 4)])
def test_product(lib, over):
    at = {**AT, **over}
    assert lib.laud_matmul_e4m3(vp(at["a"]), 256, vp(at["sa"]), vp(at["b"]), 256, vp(at["sb"]), 3, 64, 256, vp(at["out"]), 256, B.F32,
                                None, 0, None) == B.ERR_INVALID_ARG


def moe(lib, **over):  # 3 tokens, 2 of 4 experts of 128 x 256 in 8 bits
    at = {**AT, **over}
    p = B.MoeLayer(128, 256, 4, 2, B.BF16, B.E4M3, at["router"], at["up"], at["down"], at["s_up"], at["s_down"], 1, 1.0)
    return lib.laud_moe(C.byref(p), 3, vp(at["x"]), 256, vp(at["keep"]), vp(at["out"]), 256, vp(at["experts"]), vp(at["weights"]), vp(at["ws"]),
                        L.moe_workspace(p, 3), None)


SIZES = dict(router=4 * 128 * 2, up=4 * 2 * 256 * 128, down=4 * 128 * 256, s_up=4 * 2 * 2 * 4, s_down=4 * 2 * 4, keep=3, experts=24, weights=24)


@pytest.mark.parametrize("name", SIZES)
@pytest.mark.parametrize("result", ["out", "experts", "weights", "ws"])
@pytest.mark.parametrize("end", [False, True])
def test_experts(lib, result, name, end):
    if result != name:
        assert moe(lib, **{result: AT[name] if not end else AT[name] + (SIZES[name] - 1) // 16 * 16}) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("over", [dict(ws=AT["x"] + 512), dict(ws=AT["out"]), dict(experts=AT["x"] + 512 + 252), dict(weights=AT["out"] + 1024),
                                  dict(experts=AT["ws"] + 256), dict(weights=AT["x"])])
def test_experts_rows(lib, over):
    assert moe(lib, **over) == B.ERR_INVALID_ARG


def test_a_range_between_rows(tmp_path):
    """Every position of a dense range around rows that are further apart than they are long, against the bytes themselves."""
    (tmp_path / "meet.hip").write_text('#include "laud_token.h"\nextern "C" int meet(long long p, long long n, long long a, long long ld, int rows, int cols) {\n'
                                       '  return laud::range_meets_rows((void*)p, n, (void*)a, ld, 2, rows, cols);\n}\n')
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.FLAGS, "--cuda-host-only", "-shared", str(tmp_path / "meet.hip"),
                    "-o", str(tmp_path / "meet.so")], check=True, capture_output=True)
    meet = C.CDLL(str(tmp_path / "meet.so")).meet
    meet.argtypes = [C.c_longlong] * 4 + [C.c_int] * 2
    for ld, rows, cols in ((8, 3, 8), (16, 3, 8), (24, 1, 8), (13, 4, 5)):
        taken = np.zeros(400, bool)
        for r in range(rows):
            taken[100 + r * ld * 2: 100 + r * ld * 2 + cols * 2] = True
        for n in (1, 3, 8, 17, 40, 200):
            for p in range(1, 200):
                assert meet(p, n, 100, ld, rows, cols) == int(taken[p:p + n].any()), (ld, rows, cols, p, n)
        assert meet(0, 8, 100, ld, rows, cols) == 0  # (null: nothing there)
