"""Lists of rows longer than one launch has workgroups for: a workgroup goes from row to row, with the next row's loads and mask ahead of
this row's stores.  A row's result depends on nothing but the row, so a long list has to give, bit for bit, what its pieces of one
row a workgroup give, which test_gpu_token_ops.py holds against 64 bits."""
import numpy as np
import pytest
import torch

import paper_2308_15949_amd as L

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
BITS = {torch.bfloat16: torch.int16, torch.float32: torch.int32, E4M3: torch.uint8}


def equal(a, b):
    return torch.equal(a.contiguous().view(BITS[a.dtype]), b.contiguous().view(BITS[b.dtype]))


def wide_rows(n, c, extra, dtype, g=None):
    t = torch.empty(n, c + extra, device="cuda", dtype=torch.float32).fill_(float("nan"))
    if g is not None:
        t[:, :c] = torch.randn(n, c, generator=g, device="cuda")
    return t.to(dtype)[:, :c]


# channels, rows of one launch's workgroups (each one row), threads a row
@pytest.mark.parametrize("C,once", [(264, 16384), (1016, 16384), (1544, 4096), (2056, 4096), (4104, 2048), (8200, 1024), (16392, 1024)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind,z_type", [("layer", "same"), ("rms", "e4m3")])
@pytest.mark.parametrize("in_place", [False, True])
def test_a_long_list_is_its_pieces(C, once, dtype, kind, z_type, in_place):
    rows = 2 * once + once // 2 + 3
    g = torch.Generator(device="cuda").manual_seed(C)
    v = [1 + 0.2 * torch.randn(C, generator=g, device="cuda") for _ in range(2)]
    b = [0.3 * torch.randn(C, generator=g, device="cuda") if kind == "layer" else None for _ in range(2)]
    p = L.make_norm_block(C, dtype, kind, 1e-5, v[0], b[0], v[1], b[1], 0.75, 0.5)
    x, y = wide_rows(rows, C, 8, dtype, g), wide_rows(rows, C, 16, dtype, g)
    keep = torch.from_numpy(np.random.default_rng(C).integers(0, 2, rows).astype(np.uint8)).cuda()
    y.masked_fill_(keep[:, None] == 0, float("nan"))          # (a skipped row's y is not read)
    per = 7
    gate = torch.randn(-(-rows // per), C, generator=g, device="cuda")
    zt = E4M3 if z_type == "e4m3" else dtype

    def results():
        zs = torch.full((rows, -(-C // 128)), -1.0, device="cuda") if z_type == "e4m3" else None
        return wide_rows(rows, C, 8, dtype), wide_rows(rows, C, 8, zt), zs  # (pieces start at multiples of 16 bytes)

    # pieces of whole groups of rows that share a gate
    out, z, zs = results()
    each = once // per * per
    for i in range(0, rows, each):
        s = slice(i, min(i + each, rows))
        L.laud_norm_residual(p, x[s], y[s], keep[s], gate[i // per:], per, out[s], z[s], None if zs is None else zs[s])
    long_out, long_z, long_zs = results()
    if in_place:
        long_out = x
    L.laud_norm_residual(p, x, y, keep, gate, per, long_out, long_z, long_zs)
    assert equal(long_out, out) and equal(long_z, z)
    assert zs is None or equal(long_zs, zs)
    assert bool(out.isfinite().all() and z.float().isfinite().all())


@pytest.mark.parametrize("C,once", [(8, 16384), (264, 16384), (1544, 4096), (8200, 1024)])
@pytest.mark.parametrize("kept", [0, 1])
def test_all_rows_kept_or_none(C, once, kept):
    """... and the norm before a block alone, without a block's result."""
    rows = 2 * once + 5
    g = torch.Generator(device="cuda").manual_seed(C)
    w = 1 + 0.2 * torch.randn(C, generator=g, device="cuda")
    p = L.make_norm_block(C, torch.bfloat16, "rms", 1e-5, w, None, w)
    x, y = (torch.randn(rows, C, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    keep = torch.full((rows,), kept, dtype=torch.uint8, device="cuda")
    got = [torch.zeros_like(x) for _ in range(4)]
    L.laud_norm_residual(p, x, y, keep, None, 0, got[0], got[1])
    for i in range(0, rows, once):
        s = slice(i, min(i + once, rows))
        if kept:
            L.laud_norm_residual(p, x[s], y[s], None, None, 0, got[2][s], got[3][s])
        else:
            L.laud_norm_residual(p, x[s], z=got[3][s])
            got[2][s] = x[s]
    assert equal(got[0], got[2]) and equal(got[1], got[3])
    alone = torch.zeros_like(x)
    L.laud_norm_residual(p, x, z=alone)
    if not kept:
        assert equal(alone, got[1])


def test_a_long_list_against_64_bits():
    from test_gpu_token_ops import norm_case
    keep = np.random.default_rng(3).integers(0, 2, 10300)
    norm_case(10300, 1544, torch.float32, "layer", 1, bias=True, keep=keep, per=7, extra=8, inplace=True)
    norm_case(2600, 8200, torch.bfloat16, "layer", 2, bias=True, keep=keep[:2600], z="e4m3", extra=16)
