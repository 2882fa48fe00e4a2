"""Which memory the token operators touch, checked on the CPU as in test_memory_bounds.py: their kernels are built for the host and run
with every operand and workspace between two pages that nobody may touch, rows further apart than they are long, sizes that end inside
every piece, block and tile."""
import ctypes as C
import re

import numpy as np
import pytest

from paper_2308_15949_amd import binding as B
from test_memory_bounds import Call, in_a_process_of_its_own, lib  # noqa: F401  (lib: the fixture that builds the sources for the host)

BYTES = {B.F32: 4, B.BF16: 2, B.E4M3: 1}


def blocks(n):
    return -(-n // 128)


def rows(call, n, c, dtype, extra=0):
    """[n][c] rows, `extra` elements apart, the last one ending with the buffer (16-byte aligned rows: the page behind it follows)."""
    ld, eb = c + extra, BYTES[dtype]
    nbytes = ((n - 1) * ld + c) * eb
    if dtype == B.F32:
        data = call.rng.standard_normal(nbytes // 4, dtype=np.float32)
    else:
        data = call.rng.integers(0, 1 << 16 if dtype == B.BF16 else 1 << 7, nbytes // eb).astype(np.uint16 if dtype == B.BF16 else np.uint8)
    return call.buf(nbytes, data), ld


def floats(call, n):
    return call.buf(4 * n, call.rng.random(n, dtype=np.float32))


def ok(status):
    assert status == B.OK, status


def norm(call, n, c, dtype, kind, z_dtype, extra, per, in_place):
    p = B.NormBlock(c, dtype, kind, 1e-5, floats(call, c), floats(call, c), floats(call, c), floats(call, c), 1.0, 0.5)
    x, ldx = rows(call, n, c, dtype, extra)
    y, ldy = rows(call, n, c, dtype, 2 * extra)
    out, ldo = (x, ldx) if in_place else rows(call, n, c, dtype, extra)
    z, ldz = rows(call, n, c, z_dtype, extra)
    keep = call.buf(n, (call.rng.random(n) < 0.6).astype(np.uint8))
    gate = floats(call, -(-n // per) * c) if per else None
    zs = floats(call, n * blocks(c)) if z_dtype == B.E4M3 else None
    ok(call.host.laud_norm_residual(C.byref(p), n, x, ldx, y, ldy, keep, gate, per, out, ldo, z, ldz, z_dtype, zs, None))
    ok(call.host.laud_norm_residual(C.byref(p), n, x, ldx, None, 0, None, None, 0, None, 0, z, ldz, z_dtype, zs, None))


def quantize(call, n, c, dtype, block_rows, extra):
    x, ldx = rows(call, n, c, dtype, extra)
    q, ldq = rows(call, n, c, B.E4M3, 2 * extra)
    ok(call.host.laud_quantize_e4m3(x, ldx, n, c, dtype, block_rows, q, ldq, floats(call, -(-n // block_rows) * blocks(c)), None))


def matmul(call, m, n, k, dtype, extra):
    a, lda = rows(call, m, k, B.E4M3, extra)
    b, ldb = rows(call, n, k, B.E4M3, 2 * extra)
    out, ldo = rows(call, m, n, dtype, extra)
    ok(call.host.laud_matmul_e4m3(a, lda, floats(call, m * blocks(k)), b, ldb, floats(call, blocks(n) * blocks(k)), m, n, k, out, ldo, dtype,
                                  None, 0, None))


def moe(call, t, c, f, e, k, dtype, w_dtype, extra, keep, outputs):
    x, ldx = rows(call, t, c, dtype, extra)
    out, ldo = rows(call, t, c, dtype, 2 * extra)
    router, up, down = (rows(call, r, q, d)[0] for r, q, d in ((e, c, dtype), (e * 2 * f, c, w_dtype), (e * c, f, w_dtype)))
    s = [floats(call, e * 2 * blocks(f) * blocks(c)), floats(call, e * blocks(c) * blocks(f))] if w_dtype == B.E4M3 else [None, None]
    p = B.MoeLayer(c, f, e, k, dtype, w_dtype, router, up, down, *s, 1, 1.0)
    gate = call.buf(t, (call.rng.random(t) < 0.5).astype(np.uint8)) if keep else None
    nbytes = B.moe_workspace(p, t)
    ws = call.buf(nbytes)
    C.memset(ws, 0x7b, nbytes)
    ids, wt = (call.buf(4 * t * k), call.buf(4 * t * k)) if outputs else (None, None)
    ok(call.host.laud_moe(C.byref(p), t, x, ldx, gate, out, ldo, ids, wt, ws, nbytes, None))
    if outputs:
        got = np.ctypeslib.as_array((C.c_int32 * (t * k)).from_address(ids)).reshape(t, k)
        assert all((r == -1).all() or (len(set(r)) == k and (r >= 0).all() and (r < e).all() and (np.sort(r) == r).all()) for r in got)


CASES = {
    # one and two pieces a thread, one to sixteen waves a row, four pieces at the widest
    "norm_wave": (norm, 9, 264, B.BF16, B.NORM_RMS, B.E4M3, 8, 2, False),
    "norm_wave_two": (norm, 5, 1016, B.F32, B.NORM_LAYER, B.F32, 16, 1, True),
    "norm_256": (norm, 3, 1032, B.BF16, B.NORM_LAYER, B.BF16, 8, 3, True),
    "norm_256_two": (norm, 2, 4088, B.F32, B.NORM_RMS, B.E4M3, 8, 0, False),
    "norm_512": (norm, 2, 4104, B.BF16, B.NORM_RMS, B.E4M3, 24, 2, False),
    "norm_1024": (norm, 2, 8200, B.BF16, B.NORM_LAYER, B.BF16, 8, 0, True),
    "norm_1024_four": (norm, 2, 16392, B.F32, B.NORM_LAYER, B.E4M3, 8, 1, False),
    "norm_one_piece": (norm, 1, 8, B.BF16, B.NORM_RMS, B.E4M3, 0, 1, False),
    "quantize_rows": (quantize, 7, 392, B.BF16, 1, 8),
    "quantize_rows_f32": (quantize, 33, 8, B.F32, 1, 16),
    "quantize_square": (quantize, 130, 264, B.F32, 128, 8),
    "quantize_square_small": (quantize, 1, 120, B.BF16, 128, 0),
    # every tile; sizes that end inside it, reductions of one block and less, of odd and even numbers of them
    "matmul_few_rows": (matmul, 13, 40, 1168, B.BF16, 16),
    "matmul_one": (matmul, 1, 8, 16, B.F32, 0),
    "matmul_64x32": (matmul, 70, 72, 16, B.BF16, 16),
    "matmul_64x32_blocks": (matmul, 129, 40, 1456, B.F32, 16),
    "matmul_64x32_long": (matmul, 17, 136, 1680, B.BF16, 32),
    "matmul_64x32_f32": (matmul, 65, 8, 272, B.F32, 16),
    "matmul_64x32_long_f32": (matmul, 17, 136, 2064, B.F32, 32),
    "matmul_64x64": (matmul, 1000, 600, 144, B.BF16, 16),
    "matmul_64x64_long": (matmul, 1000, 600, 1424, B.BF16, 32),
    "matmul_64x64_f32": (matmul, 1000, 600, 272, B.F32, 16),
    "matmul_64x64_long_f32": (matmul, 1000, 600, 1296, B.F32, 32),
    "matmul_64x128": (matmul, 1000, 1496, 400, B.BF16, 16),
    "matmul_64x128_f32": (matmul, 1000, 1496, 400, B.F32, 16),
    "matmul_128x128": (matmul, 1800, 2040, 272, B.BF16, 16),
    "matmul_128x128_f32": (matmul, 1800, 2040, 144, B.F32, 16),
    "matmul_128x256": (matmul, 2010, 4056, 400, B.BF16, 16),
    "matmul_256x256": (matmul, 4000, 4008, 272, B.BF16, 16),
    # more entries than experts and fewer, an expert with more than sixteen tokens, widths that end inside a block, none kept
    "moe_bf16": (moe, 5, 144, 80, 4, 2, B.BF16, B.BF16, 8, False, True),
    "moe_f32": (moe, 3, 136, 24, 20, 3, B.F32, B.F32, 8, True, False),
    "moe_e4m3": (moe, 7, 272, 144, 6, 2, B.BF16, B.E4M3, 8, True, True),
    "moe_one_token_e4m3": (moe, 1, 16, 16, 3, 1, B.BF16, B.E4M3, 0, False, True),
    "moe_one_token": (moe, 1, 40, 264, 5, 3, B.BF16, B.BF16, 8, False, True),
    "moe_one_token_f32": (moe, 1, 24, 1160, 5, 4, B.F32, B.F32, 0, False, False),
    "moe_one_token_long_e4m3": (moe, 1, 144, 2064, 9, 8, B.BF16, B.E4M3, 8, False, True),
    "moe_one_token_dropped": (moe, 1, 24, 8, 5, 4, B.F32, B.F32, 0, True, True),
    "moe_one_expert": (moe, 37, 40, 8, 1, 1, B.BF16, B.BF16, 8, False, True),
    "moe_many_experts": (moe, 2, 24, 8, 1024, 32, B.F32, B.F32, 0, False, True),
    "moe_two_rounds": (moe, 70, 72, 40, 3, 2, B.BF16, B.BF16, 8, True, True),
}
# The tiles that a case is there for: rows x columns of a workgroup and the stages in LDS.
REACHES = {
    "matmul_few_rows": "k_mm8_split<unsigned short>", "matmul_one": "k_mm8_split<float>",
    "matmul_64x32": "k_mm8_tile<unsigned short, 64, 32, 32, 32, 2, 2>", "matmul_64x32_long": "k_mm8_tile<unsigned short, 64, 32, 32, 32, 3, 4>",
    "matmul_64x32_f32": "k_mm8_tile<float, 64, 32, 32, 32, 2, 2>", "matmul_64x32_long_f32": "k_mm8_tile<float, 64, 32, 32, 32, 3, 4>",
    "matmul_64x64": "k_mm8_tile<unsigned short, 64, 64, 32, 32, 2, 2>", "matmul_64x64_long": "k_mm8_tile<unsigned short, 64, 64, 32, 32, 4, 2>",
    "matmul_64x64_f32": "k_mm8_tile<float, 64, 64, 32, 32, 2, 2>", "matmul_64x64_long_f32": "k_mm8_tile<float, 64, 64, 32, 32, 4, 2>",
    "matmul_64x128": "k_mm8_tile<unsigned short, 64, 128, 32, 64, 3, 2>", "matmul_64x128_f32": "k_mm8_tile<float, 64, 128, 32, 64, 3, 2>",
    "matmul_128x128": "k_mm8_tile<unsigned short, 128, 128, 64, 64, 2, 2>", "matmul_128x128_f32": "k_mm8_tile<float, 128, 128, 64, 64, 4, 1>",
    "matmul_128x256": "k_mm8_tile<unsigned short, 128, 256, 64, 64, 3, 1>", "matmul_256x256": "k_mm8_tile<unsigned short, 256, 256, 128, 64, 2, 1>",
}


def test_every_tile_has_a_case(lib):  # noqa: F811
    import subprocess
    symbols = subprocess.run(["nm", "-C", lib], check=True, capture_output=True, text=True).stdout
    assert set(re.findall(r"k_mm8_\w+<[\w, ]+>", symbols)) == set(REACHES.values())


@pytest.mark.parametrize("front", [0, 1])
@pytest.mark.parametrize("name", CASES)
def test_kernels_stay_inside_their_buffers(lib, name, front, capfd):  # noqa: F811
    def body():
        f, *args = CASES[name]
        call = Call(lib, front)
        f(call, *args)
        assert REACHES.get(name, "") in call.launched(), call.launched()
    in_a_process_of_its_own(body, capfd)
