"""Which memory the attention kernels touch, checked on the CPU as in test_token_memory.py: every operand, index array, cache and
workspace between two pages that nobody may touch; sequences of every length from none on, rows behind the last one, pages that are
none, lengths past the table and below the new tokens, offsets that are out of order."""
import ctypes as C
import re
import subprocess

import numpy as np
import pytest

from paper_2308_15949_amd import binding as B
from test_memory_bounds import Call, in_a_process_of_its_own, lib  # noqa: F401  (lib: the fixture that builds the sources for the host)
from test_token_memory import floats, ok, rows


def ints(call, values):
    a = np.asarray(values, np.int32)
    return call.buf(a.nbytes, a)


def offsets_of(new, start=0):
    return np.concatenate(([start], start + np.cumsum(new)))


def attention(call, new, T, heads, kv_heads, D, dtype, causal, extra, keep, offsets=None, in_place=False):
    p = B.Heads(heads, kv_heads, D, dtype, causal, 0.1)
    q, ldq = rows(call, T, heads * D, dtype, extra)
    k, ldk = rows(call, T, kv_heads * D, dtype, 2 * extra)
    v, ldv = rows(call, T, kv_heads * D, dtype, 3 * extra)
    out, ldo = (q, ldq) if in_place else rows(call, T, heads * D, dtype, extra)
    offs = offsets_of(new) if offsets is None else offsets
    kept = call.buf(T, (call.rng.random(T) < 0.5).astype(np.uint8)) if keep else None
    ok(call.host.laud_attention(C.byref(p), len(offs) - 1, ints(call, offs), T, q, ldq, k, ldk, v, ldv, kept, out, ldo, None))


def cache_and_batch(call, new, lens, kv_heads, D, cache, page, table_ld, prefix_len, offsets, bad_pages):
    pages = sum(-(-max(n, 0) // page) for n in lens) + -(-prefix_len // page) + 1
    k, v = (rows(call, pages * kv_heads * page, D, cache)[0] for _ in range(2))
    s = [floats(call, pages * kv_heads * page) for _ in range(2)] if cache == B.E4M3 else [None, None]
    c = B.Cache(pages, page, kv_heads, D, cache, k, v, *s)
    order = call.rng.permutation(pages)
    shared = -(-prefix_len // page)
    table, at = np.full((len(lens), table_ld), -1), shared
    for b, n in enumerate(lens):
        need = min(-(-max(n, 0) // page), table_ld)
        table[b, :need] = order[at:at + need]
        at += need
    if bad_pages:
        table[:, ::3] = [[pages], [-5], [2 ** 31 - 1]][len(new) % 3]
    offs = offsets_of(new) if offsets is None else offsets
    b = B.Batch(len(lens), table_ld, ints(call, offs), ints(call, lens), ints(call, table), ints(call, order[:shared]) if shared else None, prefix_len)
    return c, b


def cached(call, new, lens, T, heads, kv_heads, D, dtype, cache, page, extra=0, prefix_len=0, causal=1, offsets=None, bad_pages=False, spare=2):
    longest = max([-(-max(n, 0) // page) for n in lens] + [1])
    c, b = cache_and_batch(call, new, lens, kv_heads, D, cache, page, max(longest + spare, 1), prefix_len, offsets, bad_pages)
    k, ldk = rows(call, T, kv_heads * D, dtype, extra)
    v, ldv = rows(call, T, kv_heads * D, dtype, 2 * extra)
    ok(call.host.laud_cache_write(C.byref(c), C.byref(b), T, k, ldk, v, ldv, dtype, None))
    p = B.Heads(heads, kv_heads, D, dtype, causal, 0.1)
    q, ldq = rows(call, T, heads * D, dtype, extra)
    out, ldo = rows(call, T, heads * D, dtype, 2 * extra)
    n = call.host.laud_cache_attention_workspace(C.byref(p), C.byref(c), C.byref(b), T)
    ws = call.buf(max(n, 16))  # (one that the call does not need is left alone)
    C.memset(ws, 0x7b, max(n, 16))
    if dtype == cache or dtype == B.BF16:
        ok(call.host.laud_cache_attention(C.byref(p), C.byref(c), C.byref(b), T, q, ldq, out, ldo, ws, max(n, 16), None))
    assert n or C.string_at(ws, 16) == b"\x7b" * 16
    ok(call.host.laud_cache_read(C.byref(c), C.byref(b), T, k, ldk, v, ldv, dtype, None))


F, H, E = B.F32, B.BF16, B.E4M3
CASES = {
    # every width of a tile, sequences that end inside it, of one token and none, tokens behind the last one
    "attend_bf16": (attention, [5, 0, 130, 1, 64], 203, 4, 2, 128, H, 1, 8, False),
    "attend_bf16_64": (attention, [129, 63, 1], 193, 3, 3, 64, H, 0, 0, True),
    "attend_bf16_80": (attention, [200], 200, 8, 1, 80, H, 1, 8, True),
    "attend_bf16_8": (attention, [70, 3], 80, 2, 1, 8, H, 1, 24, False, None, True),
    "attend_f32": (attention, [33, 129, 0, 2], 170, 2, 2, 128, F, 1, 8, True),
    "attend_f32_40": (attention, [1, 96, 31], 128, 5, 1, 40, F, 0, 0, False, None, True),
    "attend_many": (attention, [2] * 70 + [0] * 70 + [1], 141, 1, 1, 64, H, 1, 0, False),
    "attend_odd_offsets": (attention, [], 150, 2, 1, 64, H, 1, 0, True, [140, 20, -7, 400, 90, 130]),
    # many rows: every width of a tile in LDS, causal and not, masked, rows further apart, in place
    "tiles_bf16_8": (attention, [70, 0, 3], 75, 128, 1, 8, H, 1, 8, False),
    "tiles_bf16_8_kept": (attention, [70, 0, 3], 75, 128, 1, 8, H, 0, 8, True),
    "tiles_bf16_40": (attention, [129, 1], 133, 64, 2, 40, H, 0, 0, False, None, True),
    "tiles_bf16_40_kept": (attention, [129, 1], 133, 64, 2, 40, H, 0, 0, True, None, True),
    "tiles_bf16_72": (attention, [130], 131, 64, 1, 72, H, 1, 24, False),
    "tiles_bf16_72_kept": (attention, [130], 131, 64, 1, 72, H, 1, 24, True),
    "tiles_bf16_128": (attention, [65, 66], 131, 64, 8, 128, H, 1, 8, False, None, True),
    "tiles_bf16_128_kept": (attention, [65, 166], 235, 64, 8, 128, H, 1, 8, True, None, True),
    "tiles_f32_32": (attention, [100, 33], 140, 216, 1, 32, F, 1, 8, False),
    "tiles_f32_32_kept": (attention, [100, 33], 140, 216, 1, 32, F, 1, 8, True),
    "tiles_f32_64": (attention, [131], 132, 216, 2, 64, F, 0, 0, False),
    "tiles_f32_64_kept": (attention, [131], 132, 216, 2, 64, F, 0, 0, True),
    "tiles_f32_96": (attention, [70, 64], 134, 216, 1, 96, F, 1, 0, False),
    "tiles_f32_96_kept": (attention, [70, 64], 134, 216, 1, 96, F, 1, 0, True),
    "tiles_f32_120": (attention, [33, 98], 131, 216, 4, 120, F, 0, 8, False),
    "tiles_f32_120_kept": (attention, [33, 98], 131, 216, 4, 120, F, 0, 8, True),
    "tiles_bf16_64_odd_offsets": (attention, [], 150, 64, 1, 64, H, 1, 0, False, [140, 20, -7, 400, 90, 130]),
    "tiles_bf16_64_odd_offsets_kept": (attention, [], 150, 64, 1, 64, H, 1, 0, True, [140, 20, -7, 400, 90, 130]),
    # a list of kept rows that goes round in its ring
    "tiles_bf16_64_long_kept": (attention, [4300], 4301, 2, 1, 64, H, 0, 0, True),
    # caches of every type and page, one new token and many, parts and none
    "cached_bf16": (cached, [1, 1, 1], [300, 1, 17], 3, 8, 2, 128, H, H, 16),
    "cached_bf16_tail": (cached, [1, 3, 0, 2], [63, 64, 100, 2], 9, 4, 4, 64, H, H, 32, 8),
    "cached_bf16_rows": (cached, [40, 25], [190, 25], 70, 4, 1, 128, H, H, 64, 8),
    "cached_bf16_many_rows": (cached, [150, 20], [150, 400], 170, 4, 1, 80, H, H, 256, 0),
    "cached_bf16_tiles": (cached, [70, 60], [260, 60], 133, 16, 1, 128, H, H, 16, 8),
    "cached_bf16_tiles_64": (cached, [66], [300], 66, 32, 2, 40, H, H, 64, 0, 33),
    "cached_bf16_tiles_whole": (cached, [66], [90], 66, 16, 1, 64, H, H, 32, 0, 0, 0),
    "cached_bf16_tiles_bad": (cached, [130], [200], 131, 8, 1, 64, H, H, 16, 0, 0, 1, None, True),
    "cached_bf16_tiles_short": (cached, [70, 70], [12, -4], 140, 16, 1, 64, H, H, 16),
    "cached_bf16_tiles_prefix": (cached, [70, 66], [90, 70], 137, 16, 2, 64, H, H, 16, 8, 300),
    "cached_joined_by_eights": (cached, [100, 37], [640, 500], 138, 31, 31, 8, F, F, 128),
    "cached_e4m3": (cached, [1, 1], [513, 40], 2, 16, 2, 128, H, E, 128),
    "cached_e4m3_rows": (cached, [30, 9], [200, 9], 39, 3, 1, 48, H, E, 16, 8),
    "cached_e4m3_many_rows": (cached, [90], [700], 90, 5, 1, 128, H, E, 32),
    "cached_f32": (cached, [1, 2], [150, 33], 3, 6, 2, 128, F, F, 16, 8),
    "cached_f32_rows": (cached, [17, 40], [17, 90], 57, 2, 2, 24, F, F, 64),
    "cached_f32_e4m3_rows_only": (cached, [17, 40], [17, 90], 57, 2, 2, 32, F, E, 64),
    "cached_prefix": (cached, [1, 1, 1, 2], [20, 0, 1, 70], 6, 8, 2, 128, H, H, 16, 8, 600),
    "cached_prefix_e4m3": (cached, [2] * 9, [31] * 9, 18, 10, 2, 64, H, E, 64, 0, 1000),
    "cached_prefix_f32": (cached, [3, 3], [5, 3], 6, 4, 1, 40, F, F, 16, 0, 37),
    "cached_whole": (cached, [4, 1], [50, 3], 5, 4, 2, 64, H, H, 16, 0, 0, 0),
    # lengths below the new tokens' number, negative ones, past the table; pages that are none
    "cached_short_lens": (cached, [4, 5, 2, 1], [2, -3, 0, 1], 12, 4, 2, 64, H, H, 16),
    "cached_past_table": (cached, [2, 2], [700, 500], 4, 4, 2, 64, H, E, 16, 0, 0, 1, None, False, -30),
    "cached_bad_pages": (cached, [2, 1], [200, 90], 3, 4, 2, 128, H, H, 16, 0, 0, 1, None, True),
    "cached_bad_pages_e4m3": (cached, [2, 1, 1], [200, 90, 5], 4, 4, 2, 64, H, E, 16, 0, 40, 1, None, True),
    "cached_bad_pages_f32": (cached, [2], [200], 2, 4, 2, 64, F, F, 32, 0, 0, 1, None, True),
    "cached_odd_offsets": (cached, [], [100, 40, 30], 20, 2, 1, 64, H, H, 16, 0, 0, 1, [15, 3, 90, -2]),
    "cached_many": (cached, [1, 0] * 70, [9, 3] * 70, 75, 2, 1, 64, H, H, 16),
}


# The kernels that a case is there for: type, channels multiplied, whether keys are all rows, the kept ones or a cache's.
def reached(name, case):
    if name.startswith("tiles_"):
        return f"k_attend<{'unsigned short' if case[6] == H else 'float'}, {-(-case[5] // 32) * 32}, {int(case[9])}>"
    return f"k_attend<unsigned short, {64 if case[6] <= 64 else 128}, 2>" if name.startswith("cached_bf16_tiles") and "whole" not in name and "short" not in name else ""


REACHES = {name: kernel for name, case in CASES.items() if (kernel := reached(name, case))}


def test_every_tile_has_a_case(lib):  # noqa: F811
    symbols = subprocess.run(["nm", "-C", lib], check=True, capture_output=True, text=True).stdout
    assert set(re.findall(r"k_attend<[\w, ]+>", symbols)) == set(REACHES.values()) - {""}


@pytest.mark.parametrize("front", [0, 1])
@pytest.mark.parametrize("name", CASES)
def test_kernels_stay_inside_their_buffers(lib, name, front, capfd):  # noqa: F811
    def body():
        f, *args = CASES[name]
        call = Call(lib, front)
        f(call, *args)
        assert REACHES.get(name, "") in call.launched(), call.launched()
    in_a_process_of_its_own(body, capfd)
