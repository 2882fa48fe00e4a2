"""CPU checks of the attention operators: refusals come back as codes before anything is launched, struct layouts, workspace sizes, the
binding's checks."""
import ctypes as C
import os

import pytest

import paper_2308_15949_amd as L
from paper_2308_15949_amd import binding as B

vp = C.c_void_p
BAD, UNSUP = B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED
AT = {n: (i + 1) << 40 for i, n in enumerate(("q", "k", "v", "out", "offsets", "keep", "ck", "cv", "ks", "vs", "lens", "table", "prefix", "ws"))}


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2308_15949_amd import build
        build.build(verbose=False)
    return L.load()


def test_struct_layouts():
    assert C.sizeof(B.Heads) == 24 and C.sizeof(B.Cache) == 24 + 32 and C.sizeof(B.Batch) == 8 + 32 + 8


def heads(**over):
    f = dict(heads=4, kv_heads=2, D=64, dtype=B.BF16, causal=1, scale=0.125)
    f.update({k: v for k, v in over.items() if k in f})
    return B.Heads(*f.values())


def attention(lib, B_=2, T=6, ldq=256, ldk=128, ldv=128, ldo=256, **over):
    at = {**AT, **{k: v for k, v in over.items() if k in AT}}
    return lib.laud_attention(C.byref(heads(**over)), B_, vp(at["offsets"]), T, vp(at["q"]), ldq, vp(at["k"]), ldk, vp(at["v"]), ldv,
                              vp(at["keep"]), vp(at["out"]), ldo, None)


def test_heads_refusals(lib):
    for over in (dict(heads=0), dict(kv_heads=0), dict(heads=-4), dict(heads=3), dict(D=0), dict(D=-8), dict(dtype=B.E4M3), dict(dtype=7),
                 dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3.4e38)):
        assert attention(lib, **over) == BAD, over
    assert attention(lib, D=60) == UNSUP and attention(lib, D=136, ldq=1024, ldk=512, ldv=512, ldo=1024) == UNSUP
    assert attention(lib, heads=65536, kv_heads=1, D=8, ldq=1 << 20, ldo=1 << 20) == UNSUP
    assert lib.laud_attention(None, 1, vp(4), 1, vp(16), 256, vp(16), 128, vp(16), 128, None, vp(16), 256, None) == BAD


def test_attention_refusals(lib):
    assert attention(lib, T=0) == B.OK and attention(lib, B_=0) == B.OK and attention(lib, T=-1) == BAD and attention(lib, B_=-1) == BAD
    for k in ("q", "k", "v", "out", "offsets"):
        assert attention(lib, **{k: None}) == BAD, k
        assert attention(lib, **{k: AT[k] + 2}) == BAD, k
    assert attention(lib, ldq=248) == BAD and attention(lib, ldk=64) == BAD and attention(lib, ldv=132) == BAD and attention(lib, ldo=-256) == BAD
    assert attention(lib, T=(1 << 30) + 1, heads=1, kv_heads=1, D=8) == UNSUP
    far = (1 << 22) + 8
    assert attention(lib, ldq=far) == UNSUP and attention(lib, ldk=far) == UNSUP and attention(lib, ldv=far) == UNSUP and attention(lib, ldo=far) == UNSUP
    # results over what the call reads
    row = 512
    for name, n in (("q", row * 6), ("k", 256 * 6), ("v", 256 * 6), ("offsets", 12), ("keep", 6)):
        assert attention(lib, out=AT[name] + (n - 1) // 16 * 16) == BAD, name
    assert attention(lib, out=AT["q"], ldo=512) == BAD                  # q's place with another distance of rows
    assert attention(lib, q=AT["k"] + 256, k=AT["k"], ldq=640, ldk=640, ldv=640, v=AT["k"] + 768, out=AT["k"] + 512, ldo=640) == BAD  # columns overlap


def cache(**over):
    f = dict(pages=10, page=16, kv_heads=2, D=64, cdtype=B.BF16, ck=AT["ck"], cv=AT["cv"], ks=None, vs=None)
    f.update({k: v for k, v in over.items() if k in f})
    return B.Cache(*f.values())


def batch(**over):
    f = dict(B=2, table_ld=4, offsets=AT["offsets"], lens=AT["lens"], table=AT["table"], prefix=None, prefix_len=0)
    f.update({k: v for k, v in over.items() if k in f})
    return B.Batch(*f.values())


def write(lib, T=6, ldk=128, ldv=128, dtype=B.BF16, read=False, **over):
    at = {**AT, **{k: v for k, v in over.items() if k in ("k", "v")}}
    call = lib.laud_cache_read if read else lib.laud_cache_write
    return call(C.byref(cache(**over)), C.byref(batch(**over)), T, vp(at["k"]), ldk, vp(at["v"]), ldv, dtype, None)


E = dict(cdtype=B.E4M3, ks=AT["ks"], vs=AT["vs"])


@pytest.mark.parametrize("read", [False, True])
def test_write_and_read_refusals(lib, read):
    def w(**o):
        return write(lib, read=read, **o)
    assert w(T=0) == B.OK and w(B=0) == B.OK and w(T=-1) == BAD and w(B=-1) == BAD
    for over in (dict(pages=0), dict(page=0), dict(kv_heads=0), dict(D=0), dict(cdtype=9), dict(ck=None), dict(cv=None), dict(ck=AT["ck"] + 8),
                 dict(offsets=None), dict(lens=None), dict(table=None), dict(offsets=AT["offsets"] + 2), dict(lens=AT["lens"] + 1),
                 dict(table=AT["table"] + 2), dict(table_ld=0), dict(table_ld=1 << 27), dict(k=None), dict(v=None), dict(k=AT["k"] + 8),
                 dict(ldk=120), dict(ldv=132), dict(dtype=B.E4M3), dict(dtype=B.F32), dict(cdtype=B.F32), dict(cdtype=B.E4M3),
                 dict(E, ks=None), dict(E, vs=AT["vs"] + 4)):
        assert w(**over) == BAD, over
    for over in (dict(page=24), dict(page=8), dict(page=512), dict(D=60, ldk=128), dict(D=136, ldk=272, ldv=272), dict(E, D=72, ldk=144, ldv=144),
                 dict(pages=1 << 28), dict(kv_heads=65536, ldk=1 << 23, ldv=1 << 23), dict(T=1 << 30)):
        assert w(**over) == UNSUP, over
    assert lib.laud_cache_write(None, C.byref(batch()), 1, vp(16), 128, vp(16), 128, B.BF16, None) == BAD
    assert lib.laud_cache_write(C.byref(cache()), None, 1, vp(16), 128, vp(16), 128, B.BF16, None) == BAD
    size = 10 * 16 * 2 * 64  # codes of a cache in 8 bits
    for over in (dict(k=AT["ck"] + size - 16), dict(v=AT["cv"]), dict(k=AT["ks"]), dict(v=AT["vs"] + 1264)):
        assert w(**E, **over) == BAD, over


def test_overlaps_of_what_is_written(lib):
    for over in (dict(cv=AT["ck"] + 16), dict(ks=AT["cv"]), dict(ks=AT["vs"]), dict(offsets=AT["ck"] + 4), dict(lens=AT["vs"] + 4),
                 dict(table=AT["cv"] + 20476)):
        assert write(lib, **dict(E, **over)) == BAD, over
    for over in (dict(v=AT["k"]), dict(v=AT["k"] + 16), dict(k=AT["offsets"]), dict(v=AT["lens"]), dict(k=AT["table"] + 16)):
        assert write(lib, read=True, **over) == BAD, over


def step(lib, T=2, ldq=256, ldo=256, ws=AT["ws"], wb=1 << 40, **over):
    at = {**AT, **{k: v for k, v in over.items() if k in ("q", "out")}}
    return lib.laud_cache_attention(C.byref(heads(**over)), C.byref(cache(**over)), C.byref(batch(**over)), T, vp(at["q"]), ldq, vp(at["out"]), ldo,
                                    vp(ws), wb, None)


def test_cache_attention_refusals_and_workspace(lib):
    assert step(lib, T=0) == B.OK and step(lib, B=0) == B.OK and step(lib, T=-1) == BAD
    for over in (dict(heads=3), dict(scale=0.0), dict(dtype=B.F32), dict(cdtype=B.F32), dict(E, dtype=B.F32), dict(ck=None), dict(table_ld=0),
                 dict(q=None), dict(out=None), dict(q=AT["q"] + 8), dict(ldq=128), dict(ldo=260), dict(lens=None), dict(prefix_len=-1),
                 dict(prefix_len=5), dict(prefix_len=5, prefix=AT["prefix"] + 2), dict(out=AT["ck"]), dict(out=AT["cv"] + 16 * 10 * 256 - 16),
                 dict(E, out=AT["ks"]), dict(out=AT["table"]), dict(out=AT["offsets"]), dict(out=AT["lens"]), dict(out=AT["q"] + 16),
                 dict(prefix_len=17, prefix=AT["prefix"], out=AT["prefix"])):
        assert step(lib, **over) == BAD, over
    assert step(lib, T=1 << 30) == UNSUP and step(lib, page=48) == UNSUP
    need = lambda T=2, **o: lib.laud_cache_attention_workspace(C.byref(heads(**o)), C.byref(cache(**o)), C.byref(batch(**o)), T)  # noqa: E731
    assert need() == 0 and need(T=0) == 0 and need(heads=3) == 0 and need(table_ld=0) == 0  # 64 tokens at most: one part
    long = dict(table_ld=4096, pages=10000)
    n = need(**long)
    parts = 4 * 2 * (64 + 2)  # float32 sums and two statistics a row of a part
    assert n > 2 * parts * 4 and n < (64 * parts + 256) * 4
    assert step(lib, wb=n - 1, **long) == B.ERR_WORKSPACE and step(lib, ws=None, **long) == B.ERR_WORKSPACE
    assert step(lib, ws=AT["ws"] + 8, **long) == BAD
    for other in ("q", "out", "ck", "cv", "offsets", "lens", "table"):
        assert step(lib, ws=AT[other] - 256, wb=n, **long) == BAD, other
    assert need(prefix_len=100, prefix=AT["prefix"]) > 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    h = L.make_heads(2, 2, 64, torch.float32, True)
    assert abs(h.scale - 0.125) < 1e-9
    x, i = torch.zeros(4, 128), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: L.make_heads(2, 2, 64, torch.float16, True), lambda: L.make_heads(2, 2, 0, torch.float32, True),
                 lambda: L.make_cache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64)), lambda: L.make_cache(x, x),
                 lambda: L.make_cache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64), x),
                 lambda: L.make_batch(i, i[:2], torch.zeros(2, 4, dtype=torch.int32)), lambda: L.laud_attention(h, i, x, x, x, None, x),
                 lambda: L.laud_cache_write(B.Cache(), B.Batch(), x, x), lambda: L.laud_cache_read(B.Cache(), B.Batch(), x, x),
                 lambda: L.laud_cache_attention(h, B.Cache(), B.Batch(), x, x)):
        with pytest.raises(L.LaudError):
            call()
