"""How many parts the keys of a call over a cache are shared out over, read from the workspace it asks for (CPU)."""
import ctypes as C
import os
import random

import pytest

from paper_2308_15949_amd import binding as B
from test_memory_bounds import lib as host_lib  # noqa: F401  (the fixture that builds the sources for the host)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2308_15949_amd import build
        build.build(verbose=False)
    return B.load()


def workspace(lib, seqs, T, tokens, heads=32, kv=8, D=128, page=16, cache=B.BF16, dtype=B.BF16, prefix=0):
    """tokens: those that a row of the table has room for."""
    h, c = B.Heads(heads, kv, D, dtype, 1, 0.1), B.Cache(1 << 20, page, kv, D, cache, 1 << 44, 1 << 45, 1 << 46, 1 << 47)
    b = B.Batch(seqs, tokens // page, 1 << 40, 1 << 41, 1 << 42, 1 << 43 if prefix else None, prefix)
    return lib.laud_cache_attention_workspace(C.byref(h), C.byref(c), C.byref(b), T)


def parts(lib, seqs, T, tokens, heads=32, D=128, **more):
    n = workspace(lib, seqs, T, tokens, heads=heads, D=D, **more)
    rows = T * heads
    held = n // (4 * rows * (D + 2))  # float32 sums, a maximum and a sum of each part (sums end on 256 bytes)
    assert n == 0 or 0 <= n - held * 4 * rows * (D + 2) < 256
    return held or 1


# 32 heads over 8, one new token each, tables of 32768 tokens: as many parts of 8 workgroups a sequence as stay within 1024, two where one makes less than
# four fifths of them
@pytest.mark.parametrize("seqs,want", [(1, 64), (2, 64), (7, 18), (16, 8), (17, 7), (32, 4), (33, 3), (48, 2), (63, 2), (64, 2), (65, 2), (100, 2),
                                       (102, 2), (103, 1), (127, 1), (128, 1), (200, 1)])
def test_parts_make_the_workgroups_that_are_wanted(lib, seqs, want):
    assert parts(lib, seqs, seqs, 32768) == want


# ratios that are no whole numbers: of rows and tiles, of keys, of the sums' way to memory and the keys' time
@pytest.mark.parametrize("want,case", [
    (4, dict(seqs=1, T=512, tokens=8528)),                          # 128 tiles of 128 rows: 512 workgroups; 8528 / 2048 = 4.2
    (3, dict(seqs=3, T=600, tokens=6208)),                          # 150 tiles (200 tokens a sequence fill 6.25): 3.03 of at most 2048 keys
    (2, dict(seqs=65, T=65, tokens=8192)),                          # 520 workgroups: two parts of 4096 keys ...
    (1, dict(seqs=65, T=65, tokens=4080)),                          # ... unless a part has less than 2048
    (6, dict(seqs=20, T=20, tokens=8192, heads=16, cache=B.F32, dtype=B.F32)),  # 160 workgroups: 6.4
])
def test_parts_at_ratios_between_whole_numbers(lib, want, case):
    assert parts(lib, **case) == want


def test_both_builds_share_out_alike(lib, host_lib):  # noqa: F811
    host, rng = C.CDLL(host_lib), random.Random(1)
    host.laud_cache_attention_workspace.restype = C.c_size_t
    host.laud_cache_attention_workspace.argtypes = lib.laud_cache_attention_workspace.argtypes
    several = 0
    for _ in range(3000):
        seqs, kv, cache = int(2 ** rng.uniform(0, 8)), rng.choice((1, 2, 3, 8, 12)), rng.choice((B.BF16, B.E4M3, B.F32))
        case = dict(seqs=seqs, T=seqs * int(2 ** rng.uniform(0, 9)), tokens=16 * int(2 ** rng.uniform(0, 12)), heads=kv * rng.choice((1, 3, 4, 5)), kv=kv,
                    D=rng.choice((32, 80, 128)), cache=cache, dtype=B.F32 if cache == B.F32 else B.BF16, prefix=rng.choice((0, 0, int(2 ** rng.uniform(0, 14)))))
        n = workspace(lib, **case)
        several += n > 0
        assert n == workspace(host, **case), case
    assert several > 500


def test_numbers_of_more_than_32_bits_are_refused(lib):
    """ctypes would cut them: 2^32 + 8 heads were 8."""
    import torch

    import paper_2308_15949_amd as L
    h, c, b = B.Heads(32, 8, 128, B.BF16, 1, 0.1), B.Cache(1 << 20, 16, 8, 128, B.BF16, 1 << 44, 1 << 45), B.Batch(1, 2048, 1 << 40, 1 << 41, 1 << 42)
    many = (1 << 32) + 8
    assert L.cache_attention_workspace(h, c, b, 8) > 0
    for call in (lambda: L.make_heads(many, 8, 64, torch.bfloat16, True), lambda: L.make_heads(8, many, 64, torch.bfloat16, True),
                 lambda: L.make_heads(8, 8, many, torch.bfloat16, True), lambda: L.cache_attention_workspace(h, c, b, many)):
        with pytest.raises(L.LaudError) as refusal:
            call()
        assert refusal.value.status == B.ERR_INVALID_ARG
