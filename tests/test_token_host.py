"""CPU checks of the token operators: refusals come back as codes before anything is launched, workspace sizes, struct layouts."""
import ctypes as C

import pytest

import paper_2308_15949_amd as L
from paper_2308_15949_amd import binding as B

FAKE = 0x10000  # never dereferenced: validation happens on the host before any launch
FAR = 0x10000000000
vp = C.c_void_p


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2308_15949_amd import build
        build.build(verbose=False)
    return L.load()


def test_struct_layouts():
    assert C.sizeof(B.NormBlock) == 16 + 4 * 8 + 8
    assert C.sizeof(B.MoeLayer) == 24 + 5 * 8 + 8


def norm(lib, p=None, rows=2, x=FAKE, ldx=64, y=FAR, ldy=64, keep=None, gate=None, per=0, out=2 * FAR, ldo=64, z=None, ldz=0, zt=B.F32,
         zs=None, **over):
    if p is None:
        f = dict(C=64, dtype=B.F32, kind=0, eps=1e-5, post_w=FAKE, post_b=None, pre_w=FAKE, pre_b=None, alpha=1.0, beta=1.0)
        f.update(over)
        p = B.NormBlock(*f.values())
    return lib.laud_norm_residual(C.byref(p), rows, vp(x), ldx, vp(y), ldy, vp(keep), vp(gate), per, vp(out), ldo, vp(z), ldz, zt, vp(zs), None)


def test_norm_refusals(lib):
    bad, unsup = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED
    assert norm(lib, rows=0) == B.OK and norm(lib, rows=0, x=None, out=None) == B.OK
    assert norm(lib, rows=-1) == bad
    assert lib.laud_norm_residual(None, 1, vp(FAKE), 64, None, 0, None, None, 0, vp(FAR), 64, None, 0, 0, None, None) == bad
    assert norm(lib, C=60, ldx=64) == unsup and norm(lib, C=32776, ldx=40000) == unsup and norm(lib, C=0) == bad
    assert norm(lib, dtype=B.E4M3) == bad and norm(lib, kind=2) == bad
    assert norm(lib, eps=-1.0) == bad and norm(lib, eps=float("nan")) == bad
    assert norm(lib, x=None) == bad and norm(lib, out=None) == bad           # nothing to write
    assert norm(lib, ldx=56) == bad and norm(lib, ldx=68) == bad and norm(lib, ldy=0) == bad and norm(lib, ldo=-64) == bad
    assert norm(lib, x=FAKE + 4) == bad and norm(lib, y=FAR + 8) == bad and norm(lib, post_w=FAKE + 4) == bad
    assert norm(lib, y=None, keep=FAKE) == bad and norm(lib, y=None, gate=FAKE, per=1) == bad
    assert norm(lib, gate=FAKE, per=0) == bad
    assert norm(lib, z=3 * FAR, ldz=64, pre_w=None) == bad
    assert norm(lib, z=3 * FAR, ldz=64, zt=B.BF16) == bad                     # neither x's type nor 8 bits
    assert norm(lib, z=3 * FAR, ldz=64, zt=B.E4M3) == bad                     # no scales
    assert norm(lib, out=FAKE + 256) == bad                                   # over the second row of x
    assert norm(lib, out=FAKE, ldo=128) == bad                                # x's place with another distance of rows
    assert norm(lib, z=2 * FAR, ldz=64) == bad                                # both results in one place
    assert norm(lib, rows=3, z=FAKE, ldz=64, zt=B.E4M3, zs=FAR) == bad        # narrower rows over x


def test_rows_side_by_side_are_no_overlap(lib):
    """Columns of one wider array, the same distance from row to row, share no byte: checked on the refusal of what does overlap (a
    call that passed would launch)."""
    assert norm(lib, ldx=128, out=FAKE + 128, ldo=128) == B.ERR_INVALID_ARG   # 64 float32 columns, 32 further: overlap
    assert norm(lib, ldx=96, out=FAKE + 256, ldo=96) == B.ERR_INVALID_ARG     # runs into the next row


def test_quantize_refusals(lib):
    def q(x=FAKE, ldx=64, rows=2, cols=64, dtype=B.F32, br=1, out=FAR, ldq=64, s=FAKE):
        return lib.laud_quantize_e4m3(vp(x), ldx, rows, cols, dtype, br, vp(out), ldq, vp(s), None)
    bad, unsup = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED
    assert q(rows=0) == B.OK
    assert q(rows=-1) == bad and q(cols=0) == bad and q(cols=60) == unsup and q(dtype=B.E4M3) == bad and q(br=64) == bad
    assert q(x=None) == bad and q(out=None) == bad and q(s=None) == bad and q(x=FAKE + 8) == bad and q(out=FAR + 8) == bad
    assert q(ldx=32) == bad and q(ldq=60) == bad and q(out=FAKE) == bad


def test_matmul_refusals(lib):
    def m(a=FAKE, lda=64, sa=FAKE, b=FAR, ldb=64, sb=FAKE, M=2, N=16, K=64, out=2 * FAR, ldo=16, ot=B.F32, ws=None, wb=0):
        return lib.laud_matmul_e4m3(vp(a), lda, vp(sa), vp(b), ldb, vp(sb), M, N, K, vp(out), ldo, ot, vp(ws), wb, None)
    bad, unsup = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED
    assert m(M=0) == B.OK
    assert m(M=-1) == bad and m(N=0) == bad and m(K=0) == bad and m(ot=B.E4M3) == bad
    assert m(N=12) == unsup and m(K=24, lda=32, ldb=32) == unsup
    for k in ("a", "sa", "b", "sb", "out"):
        assert m(**{k: None}) == bad
    assert m(lda=48) == bad and m(ldb=72) == bad and m(ldo=8) == bad and m(ldo=20) == bad
    assert m(a=FAKE + 8) == bad and m(out=2 * FAR + 4) == bad
    assert m(out=FAKE) == bad and m(out=FAR + 16) == bad
    assert m(lda=(1 << 22) + 16) == unsup


def moe_layer(**over):
    f = dict(C=64, F=32, E=4, top_k=2, dtype=B.BF16, w_dtype=B.BF16, router=FAKE, up=FAKE, down=FAKE, s_up=None, s_down=None, renorm=0,
             scale=1.0)
    f.update(over)
    return B.MoeLayer(*f.values())


def moe(lib, T=2, x=FAKE, ldx=64, out=FAR, ldo=64, ws=FAKE, wb=1 << 40, **over):
    return lib.laud_moe(C.byref(moe_layer(**over)), T, vp(x), ldx, None, vp(out), ldo, None, None, vp(ws), wb, None)


def test_moe_refusals_and_workspace(lib):
    bad, unsup = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED
    assert moe(lib, T=0) == B.OK and moe(lib, T=-1) == bad and moe(lib, T=B.MOE_MAX_TOKENS + 1) == unsup
    assert lib.laud_moe(None, 1, vp(FAKE), 64, None, vp(FAR), 64, None, None, vp(FAKE), 1 << 30, None) == bad
    for k in ("C", "F", "E", "top_k"):
        assert moe(lib, **{k: 0}) == bad
    assert moe(lib, top_k=5) == bad and moe(lib, E=1025) == unsup and moe(lib, E=64, top_k=33) == unsup
    assert moe(lib, C=60) == unsup and moe(lib, F=36) == unsup
    assert moe(lib, dtype=B.E4M3) == bad and moe(lib, dtype=B.F32) == bad and moe(lib, dtype=B.F32, w_dtype=B.E4M3) == unsup
    assert moe(lib, w_dtype=B.E4M3) == bad and moe(lib, w_dtype=B.E4M3, F=40, s_up=FAKE, s_down=FAKE) == unsup
    for k in ("x", "out", "router", "up", "down"):
        assert moe(lib, **{k: None}) == bad
        assert moe(lib, **{k: FAR + 8}) == bad
    assert moe(lib, ldx=56) == bad and moe(lib, ldo=68) == bad and moe(lib, out=FAKE + 128) == bad
    assert moe(lib, ws=None) == B.ERR_WORKSPACE and moe(lib, wb=16) == B.ERR_WORKSPACE and moe(lib, ws=FAKE + 8) == bad
    for T in (1, 3, 64, 1000):
        need = L.moe_workspace(moe_layer(), T)
        assert need >= T * 2 * (8 + 128 * 4) and L.moe_workspace(moe_layer(E=0), T) == 0
        assert moe(lib, T=T, wb=need - 1) == B.ERR_WORKSPACE
    assert L.moe_workspace(moe_layer(), 0) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    x = torch.zeros(2, 64)
    with pytest.raises(L.LaudError):
        L.make_norm_block(64, torch.float32, "rms", 1e-5, torch.ones(64))     # a host tensor
    with pytest.raises(L.LaudError):
        L.make_norm_block(64, torch.float16, "rms", 1e-5)
    with pytest.raises(L.LaudError):
        L.make_norm_block(64, torch.float32, "batch", 1e-5)
    with pytest.raises(L.LaudError):
        L.laud_norm_residual(L.make_norm_block(64, torch.float32, "rms", 1e-5), x, out=x)
    with pytest.raises(L.LaudError):
        L.laud_quantize_e4m3(x, x, x)
    with pytest.raises(L.LaudError):
        L.laud_matmul_e4m3(x, x, x, x, x)
