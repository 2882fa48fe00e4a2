"""Attention of a token block against a plain implementation in 64 bits: types, head layouts, widths, lengths from none to long ones,
strides, masks that leave rows empty, special values in masked places, caches of every type, prefixes, streams and graphs.

Tolerances.  eps / 2 is half a step of a type: 2^-8 in bf16, 2^-24 in float32.  A score is a sum of D products in float32, off by at most
(D + 2) 2^-24 of the sum of magnitudes, and as an exponent once more by 2^-23 of itself; an error d of the scores changes a weight
by a factor within exp(+-2 d) after the division by their sum, and sums over n keys add n 2^-24, the exponential, the parts' joins and the division 2^-20.
A weight is rounded to bf16 for bf16 values.  All of these are relative to sum_j w_j |v_j|; the result's own rounding is relative to it."""
import math

import numpy as np
import pytest
import torch

import paper_2308_15949_amd as L

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
F32, BF16 = torch.float32, torch.bfloat16
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *shape):
    return torch.randn(*shape, generator=g)


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def spread(t, extra):
    """The same rows on the device, `extra` elements further apart; what lies between them is NaN."""
    n, c = t.shape
    wide = torch.full((n, c + extra), float("nan"), dtype=F32).to(t.dtype).cuda()
    wide[:, :c] = t.cuda()
    return wide[:, :c]


def attend64(q, k, v, scale, allowed):
    """q [n][H][D], k, v [m][Hk][D] float64, allowed [n][m]: result, sum of weight * |v|, and what the scores may be off by; a value
    has no part where its key is not allowed."""
    n, H, D = q.shape
    m, Hk, _ = k.shape
    if n == 0 or m == 0:
        z = torch.zeros(n, H, D, dtype=torch.float64)
        return z, z, torch.zeros(n, H, 1, dtype=torch.float64)
    kk, vv = (x.repeat_interleave(H // Hk, 1).permute(1, 0, 2) for x in (k, v))
    qq = q.permute(1, 0, 2)
    z = scale * (qq @ kk.transpose(1, 2))
    mag = scale * (qq.abs() @ kk.abs().transpose(1, 2))
    z = torch.where(allowed, z, -math.inf)
    top = z.max(2, keepdim=True).values
    w = torch.where(allowed, torch.exp(z - torch.where(torch.isinf(top) & (top < 0), 0.0, top)), 0.0)
    total = w.sum(2, keepdim=True)
    w = torch.where(total == 0, 0.0, w / total)
    off = torch.where(allowed, mag * (D + 2) * 2.0 ** -24 + z.abs() * 2.0 ** -23, 0.0)
    off = torch.nan_to_num(off, 0.0, 0.0).max(2, keepdim=True).values
    if bool(torch.isfinite(vv).all()):
        out, size = w @ vv, w @ vv.abs()
    else:  # a NaN or an infinity reaches the rows that see it only
        out, size = (torch.stack([torch.where(allowed[i][:, None], w[:, i, :, None] * x, 0.0).sum(1) for i in range(n)], 1) for x in (vv, vv.abs()))
    return out.permute(1, 0, 2), size.permute(1, 0, 2), off.permute(1, 0, 2)


def near(got, ref, size, off, n, dtype):
    """Whether got [..][H][D] is within what its types allow; values that are no numbers have to be the same ones."""
    got = got.double().cpu()
    tol = HALF[dtype] * ref.abs() + size * (2 * off + n * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -8 if dtype == BF16 else 0.0))
    same = (got == ref) | (got.isnan() & ref.isnan())
    good = same | ((got - ref).abs() <= tol)
    if not bool(good.all()):
        bad = (~good).nonzero()
        i = tuple(bad[0].tolist())
        print(f"{len(bad)} of {good.numel()} off, first at {i}: {float(got[i])} for {float(ref[i])}, tolerance {float(tol[i])}", flush=True)
    return bool(good.all())


def offsets_of(new, start=0):
    return np.concatenate(([start], start + np.cumsum(new))).astype(int)


# ----- over the tokens of packed sequences ---------------------------------------------------------------------------------------
def attention_case(new, heads, kv, D, dtype, causal, seed, keep=None, extra=0, scale=None, start=0, behind=0, in_place=False, change=None, joined=False):
    g = gen(seed)
    offs = offsets_of(new, start)
    T = int(offs[-1]) + behind
    q, k, v = rand(g, T, heads * D).to(dtype), rand(g, T, kv * D).to(dtype), rand(g, T, kv * D).to(dtype)
    if change:
        change(q.view(T, heads, D), k.view(T, kv, D), v.view(T, kv, D))
    if joined:
        wide = spread(torch.cat((q, k, v), 1), extra)
        qd, kd, vd = wide[:, :heads * D], wide[:, heads * D:(heads + kv) * D], wide[:, (heads + kv) * D:]
    else:
        qd, kd, vd = spread(q, extra), spread(k, 2 * extra), spread(v, 3 * extra)
    out = qd if in_place else spread(torch.full_like(q, 7.0), extra)
    before = out.clone()
    kept = None if keep is None else torch.tensor(np.asarray(keep), dtype=torch.uint8)
    p = L.make_heads(heads, kv, D, dtype, causal, scale)
    L.laud_attention(p, ints(offs), qd, kd, vd, None if kept is None else kept.cuda(), out)
    torch.cuda.synchronize()
    got = out.cpu()
    for i, j in zip(offs, offs[1:]):
        n = j - i
        allowed = torch.ones(n, n, dtype=torch.bool)
        if causal:
            allowed = allowed.tril()
        if kept is not None:
            here = kept[i:j] != 0
            allowed = allowed & here[:, None] & here[None, :]
        ref = attend64(q[i:j].double().view(n, heads, D), k[i:j].double().view(n, kv, D), v[i:j].double().view(n, kv, D), p.scale, allowed)
        assert near(got[i:j].view(n, heads, D), *ref, n, dtype), (i, j)
    for i, j in ((0, offs[0]), (offs[-1], T)):  # rows of no sequence are left as they were
        assert torch.equal(got[i:j].view(torch.uint8), before[i:j].cpu().view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [8, 16, 40, 64, 72, 80, 96, 128])
def test_widths(D, dtype):
    attention_case([33, 1, 130], 4, 2, D, dtype, True, D)
    attention_case([70, 5], 2, 2, D, dtype, False, D + 1, extra=8)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 600])
def test_lengths(n, dtype):
    attention_case([n], 3, 1, 64, dtype, True, n)
    attention_case([n, 1, 0, n], 2, 1, 128, dtype, False, n + 1, extra=16, joined=True)


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 8), (8, 1), (16, 4), (5, 5), (15, 3), (40, 8)])
def test_head_layouts(heads, kv):
    for dtype in (BF16, F32):
        attention_case([100, 37], heads, kv, 64, dtype, True, heads, extra=24)
    attention_case([150], heads, kv, 128, BF16, False, kv)


def test_many_sequences_and_rows_of_none():
    g = np.random.default_rng(3)
    for dtype in (BF16, F32):
        attention_case(list(g.integers(0, 9, 150)), 2, 1, 64, dtype, True, 5, start=3, behind=70)
        attention_case([0] * 65 + [40] + [0] * 3, 2, 2, 80, dtype, False, 6, behind=1)
        attention_case([0, 0], 2, 2, 64, dtype, True, 6, behind=9)
        attention_case([129], 4, 4, 40, dtype, True, 7, start=130, behind=130)
    q = torch.zeros(0, 64, device="cuda")
    L.laud_attention(L.make_heads(1, 1, 64, F32, True), ints([0]), q, q, q, None, q)  # no sequence, no row


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_masks(dtype, causal):
    g = np.random.default_rng(4)
    for share in (0.0, 0.03, 0.5, 0.97, 1.0):
        attention_case([150, 1, 70, 64], 4, 2, 80, dtype, causal, 8, keep=g.random(285) < share, extra=8)
    first = np.ones(300)
    first[:200] = 0
    attention_case([300], 2, 1, 128, dtype, causal, 9, keep=first)
    attention_case([300], 2, 1, 64, dtype, causal, 9, keep=1 - first)
    attention_case([200], 2, 1, 64, dtype, causal, 10, keep=g.integers(0, 3, 200) * 100)  # any byte but 0 keeps


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_scales(dtype):
    attention_case([130, 60], 4, 2, 64, dtype, True, 11, in_place=True, extra=8)
    attention_case([90], 2, 2, 128, dtype, True, 12, scale=3.0)      # weights near one and zero
    attention_case([90], 2, 2, 128, dtype, False, 13, scale=1e-6)    # ... all alike
    attention_case([257], 2, 2, 64, dtype, False, 14, scale=0.125, change=lambda q, k, v: k.mul_(20))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_special_values_stay_with_who_sees_them(dtype, what):
    def put(q, k, v):
        v[70, 0, 3] = what      # seen by the tokens from 70 on
        v[100, 0, 17] = what
        v[100, 0, 18] = -what
        v[33] = what
    attention_case([129, 40], 2, 1, 64, dtype, True, 15, change=put)
    attention_case([129, 40], 2, 1, 128, dtype, True, 16, change=put)

    def keys(q, k, v):
        k[140] = math.nan       # another sequence's first token
        v[140] = what
    attention_case([140, 30], 2, 1, 80, dtype, True, 17, change=lambda q, k, v: (k[139].fill_(math.nan), v[139].fill_(what)))
    keep = np.ones(170)
    keep[[5, 66, 140]] = 0

    def masked(q, k, v):
        for t in (5, 66, 140):
            q[t], k[t], v[t] = math.nan, what, what
    attention_case([140, 30], 2, 1, 64, dtype, False, 18, keep=keep, change=masked)
    attention_case([140, 30], 2, 1, 128, dtype, True, 19, keep=keep, change=masked)
    attention_case([140, 30], 2, 1, 64, dtype, False, 20, change=keys)  # (token 140 is the second sequence's own)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_largest_and_smallest_scores(dtype):
    big = 2.0 ** 60

    def put(q, k, v):
        q[:], k[:] = big, -big  # every score -2^127 or so: still a score
    attention_case([70], 1, 1, 64, dtype, True, 21, scale=0.0625, change=put)

    def low(q, k, v):
        q[:], k[:40] = 1.0, -3.0e38   # the sum of the products is -infinity: no weight
    attention_case([70], 1, 1, 64, dtype, True, 22, scale=1.0, change=low)
    attention_case([130], 2, 2, 64, dtype, True, 23, change=lambda q, k, v: (q.zero_(), k.zero_()))
    attention_case([130], 2, 2, 64, dtype, True, 24, change=lambda q, k, v: v.mul_(2.0 ** -120))


def test_a_long_sequence():
    attention_case([5000], 2, 1, 64, BF16, True, 25)
    attention_case([3001], 1, 1, 128, F32, False, 26)


# Many rows (heads times tokens above 8192 in bf16, 28000 in float32) go through the tiles in LDS.
WIDE = {BF16: 64, F32: 192}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [8, 24, 32, 40, 64, 72, 80, 96, 104, 128])
def test_many_rows_widths(D, dtype):
    attention_case([33, 1, 130, 0, 70], WIDE[dtype], 2, D, dtype, True, D, extra=8)
    attention_case([65, 128, 3], WIDE[dtype], WIDE[dtype] // 2, D, dtype, False, D + 1, joined=True, extra=24)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n", [129, 160, 191, 192, 193, 255, 256, 257, 383, 385])
def test_many_rows_lengths(n, dtype):
    attention_case([n, 31, 1], WIDE[dtype], 4, 64, dtype, True, n)
    attention_case([n, 64], WIDE[dtype] + 4, 4, 128, dtype, False, n + 1, extra=16)   # (heads that eight do not divide)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_masks(dtype, causal):
    g = np.random.default_rng(5)
    for share in (0.0, 0.02, 0.5, 1.0):
        attention_case([150, 1, 70, 64], WIDE[dtype], 2, 80, dtype, causal, 8, keep=g.random(285) < share, extra=8)
    first = np.ones(300)
    first[:200] = 0
    attention_case([300], WIDE[dtype], 2, 64, dtype, causal, 10, keep=first)
    attention_case([300], WIDE[dtype], 2, 128, dtype, causal, 11, keep=1 - first)


@pytest.mark.parametrize("dtype,heads", [(BF16, 1), (F32, 4)])
def test_masks_of_more_than_4096_keys(dtype, heads):
    """The list of kept rows goes round."""
    g = np.random.default_rng(6)
    keep = g.random(8700) < 0.6
    keep[4000:4200] = 0
    attention_case([8500, 200], heads, 1, 64, dtype, False, 12, keep=keep)
    attention_case([8700], heads, 1, 32, dtype, True, 13, keep=keep)
    keep = g.random(9000) < 0.02
    keep[2000:5000] = 1
    attention_case([6500, 2500], heads, 1, 64, dtype, True, 14, keep=keep)
    attention_case([9000], heads, 1, 96, dtype, False, 15, keep=1 - keep)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("few", [False, True])
def test_rows_far_apart(dtype, causal, few):
    """Rows beyond 2 GiB of the first; kept ones of one step more than that from each other, and less."""
    heads, D, n = 4 if few else WIDE[dtype], 64, 420
    g = gen(30)
    wide = torch.empty(n, 1 << 22, dtype=dtype, device="cuda")
    k, v = wide[:, 8:8 + D], wide[:, -D:]
    q, kh, vh = rand(g, n, heads * D).to(dtype), rand(g, n, D).to(dtype), rand(g, n, D).to(dtype)
    k.copy_(kh)
    v.copy_(vh)
    out = torch.full((n, heads * D), 7.0, dtype=dtype, device="cuda")
    p = L.make_heads(heads, 1, D, dtype, causal)
    for share in (0.1, 0.9, 1.0):
        kept = torch.rand(n, generator=g) < share
        L.laud_attention(p, ints([0, n]), q.cuda(), k, v, kept.to(torch.uint8).cuda() if share < 1.0 else None, out)
        torch.cuda.synchronize()
        allowed = kept[:, None] & kept[None, :]
        allowed = allowed.tril() if causal else allowed
        ref = attend64(q.double().view(n, heads, D), kh.double().view(n, 1, D), vh.double().view(n, 1, D), p.scale, allowed)
        assert near(out.cpu().view(n, heads, D), *ref, n, dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_many_rows_special_values(dtype, what):
    heads = WIDE[dtype]

    def put(q, k, v):
        v[70, 0, 3] = what
        v[100, 0, 17], v[100, 0, 18] = what, -what
        v[33], v[128] = what, -what
    attention_case([129, 40], heads, 1, 64, dtype, True, 15, change=put)
    attention_case([129, 40], heads, 1, 128, dtype, True, 16, change=put)
    attention_case([140, 30], heads, 1, 80, dtype, True, 17, change=lambda q, k, v: (k[139].fill_(math.nan), v[139].fill_(what)))
    keep = np.ones(170)
    keep[[5, 66, 140]] = 0

    def masked(q, k, v):
        for t in (5, 66, 140):
            q[t], k[t], v[t] = math.nan, what, what
    attention_case([140, 30], heads, 1, 96, dtype, False, 18, keep=keep, change=masked)
    attention_case([140, 30], heads, 1, 24, dtype, True, 19, keep=keep, change=masked)
    attention_case([140, 30], heads, 1, 64, dtype, True, 20, change=lambda q, k, v: (q[3].fill_(math.nan), k[150].fill_(what)))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_in_place_strays_and_scales(dtype):
    heads = WIDE[dtype]
    attention_case([130, 60], heads, 2, 64, dtype, True, 21, in_place=True, extra=8)
    attention_case([129], heads, 2, 40, dtype, True, 22, start=130, behind=130)
    keep = np.random.default_rng(5).random(200) < 0.5
    attention_case([130, 70], heads, 2, 64, dtype, True, 28, keep=keep, in_place=True, extra=8)
    attention_case([150, 30], heads, 1, 104, dtype, False, 29, keep=keep, in_place=True, start=13, behind=7)
    attention_case(list(np.random.default_rng(3).integers(0, 9, 150)), heads, 2, 64, dtype, True, 23, start=3, behind=70)
    attention_case([190], heads, 2, 128, dtype, True, 24, scale=3.0)
    attention_case([190], heads, 2, 64, dtype, False, 25, scale=1e-6)
    # scores that grow from step to step: the sums are taken anew again and again, or not (less than 2^8)
    for by in (1.0, 0.02):
        def grow(q, k, v):
            q[:] = 1.0
            k[:] = (by * torch.arange(len(k)))[:, None, None]
        attention_case([300], heads, 2, 64, dtype, True, 26, scale=0.05, change=grow)
        attention_case([300], heads, 2, 128, dtype, False, 27, scale=0.05, change=lambda q, k, v: (grow(q, k, v), k.neg_()))


# ----- over a cache --------------------------------------------------------------------------------------------------------------
class Paged:
    """A cache of pages that belong to sequences in no order; places nobody wrote hold NaN."""

    def __init__(self, g, lens, kv, D, dtype, page, prefix=0, spare=2):
        self.kv, self.D, self.page, self.dtype = kv, D, page, dtype
        self.shared = -(-prefix // page)
        need = [-(-max(n, 0) // page) for n in lens]
        pages = self.shared + sum(need) + 3
        shape = (pages, kv, page, D)
        if dtype == E4M3:
            self.k, self.v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:3], math.nan, device="cuda") for _ in range(2))
        else:
            self.k, self.v = (torch.full(shape, math.nan, device="cuda", dtype=dtype) for _ in range(2))
            self.ks = self.vs = None
        order = torch.randperm(pages, generator=g).tolist()
        self.pages, self.prefix_pages = [], order[:self.shared]
        at = self.shared
        for n in need:
            self.pages.append(order[at:at + n])
            at += n
        wide = max(need + [0]) + spare
        self.table = ints([p + [-1] * (wide - len(p)) for p in self.pages])
        self.desc = L.make_cache(self.k, self.v, self.ks, self.vs)

    def batch(self, new, lens, prefix=0, start=0):
        return L.make_batch(ints(offsets_of(new, start)), ints(lens), self.table, ints(self.prefix_pages) if self.shared else None, prefix)

    def rows64(self, which, pages, n):
        """The first n rows of those pages as the values they stand for, [n][kv][D]."""
        x = getattr(self, which).float().cpu().double()
        if self.ks is not None:
            x = x * getattr(self, which + "s").cpu().double()[..., None]
        return x[pages].permute(0, 2, 1, 3).reshape(-1, self.kv, self.D)[:n]


def fill(cache, g, lens, prefix, dtype, change=None):
    """Keys and values of all tokens through laud_cache_write (the prefix as a sequence of its own); the rows."""
    T = sum(lens)
    k, v = (rand(g, T + prefix, cache.kv * cache.D).to(dtype) for _ in range(2))
    if change:
        change(k[prefix:].view(T, cache.kv, cache.D), v[prefix:].view(T, cache.kv, cache.D))
    if prefix:
        b = L.make_batch(ints([0, prefix]), ints([prefix]), ints([cache.prefix_pages]))
        L.laud_cache_write(cache.desc, b, k[:prefix].cuda(), v[:prefix].cuda())
    if T:
        L.laud_cache_write(cache.desc, cache.batch(lens, lens), spread(k[prefix:], 8), spread(v[prefix:], 16))
    torch.cuda.synchronize()
    return k, v


def cached_case(new, lens, heads, kv, D, dtype, cache_type, page, seed, prefix=0, causal=True, extra=0, start=0, behind=0, change=None, scale=None,
                in_place=False):
    g = gen(seed)
    cache = Paged(g, lens, kv, D, cache_type, page, prefix)
    fill(cache, g, lens, prefix, dtype, change)
    T = sum(new) + start + behind
    q = rand(g, T, heads * D).to(dtype)
    qd = spread(q, extra)
    out = qd if in_place else spread(torch.full_like(q, 7.0), 2 * extra)
    before = out.clone()
    p = L.make_heads(heads, kv, D, dtype, causal, scale)
    b = cache.batch(new, lens, prefix, start)
    n = L.cache_attention_workspace(p, cache.desc, b, T)
    ws = torch.full((max(n, 1),), 0x7b, dtype=torch.uint8, device="cuda") if n else None
    L.laud_cache_attention(p, cache.desc, b, qd, out, ws)
    torch.cuda.synchronize()
    got, offs = out.cpu(), offsets_of(new, start)
    kp, vp = (cache.rows64(x, cache.prefix_pages, prefix) for x in ("k", "v"))
    for i, (m, pages, ln) in enumerate(zip(new, cache.pages, lens)):
        k, v = (torch.cat((a, cache.rows64(x, pages, ln))) for x, a in (("k", kp), ("v", vp)))
        allowed = torch.ones(m, prefix + ln, dtype=torch.bool)
        if causal:
            allowed = torch.arange(prefix + ln)[None, :] <= (prefix + ln - m + torch.arange(m))[:, None]
            allowed[:, :prefix] = True
        rows = slice(int(offs[i]), int(offs[i + 1]))
        ref = attend64(q[rows].double().view(m, heads, D), k, v, p.scale, allowed)
        assert near(got[rows].view(m, heads, D), *ref, prefix + ln, dtype), i
    for i, j in ((0, start), (T - behind, T)):
        assert torch.equal(got[i:j].view(torch.uint8), before[i:j].cpu().view(torch.uint8))


TYPES = [(BF16, BF16), (BF16, E4M3), (F32, F32)]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 64, 127, 128, 129, 500, 2000])
def test_one_token_over_lengths(n, dtype, cache):
    cached_case([1], [n], 8, 2, 128, dtype, cache, 16, n)
    cached_case([1, 1, 1], [n, 1, n + 5], 4, 4, 64, dtype, cache, 64, n + 1, extra=8)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128])
def test_cached_widths(D, dtype, cache):
    cached_case([1, 3], [40, 200], 6, 2, D, dtype, cache, 32, D)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [8, 24, 40, 72, 104, 120])
def test_cached_widths_of_eight(D, dtype):
    cached_case([1, 3], [40, 200], 6, 2, D, dtype, dtype, 16, D)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_pages(page, dtype, cache):
    cached_case([1, 2, 1], [page, page + 1, 3 * page - 1], 4, 1, 64, dtype, cache, page, page)
    cached_case([1, 2, 1], [5, 300, 77], 4, 1, 128, dtype, cache, page, page + 1, prefix=page + 7)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new", [2, 5, 16, 17, 40, 130])
def test_several_new_tokens(new, dtype, cache):
    cached_case([new, 1, new], [new, 30, new + 333], 4, 2, 64, dtype, cache, 16, new)
    cached_case([new, 3], [new + 50, 3], 5, 1, 128, dtype, cache, 32, new, causal=False, extra=8)


@pytest.mark.parametrize("D", [8, 64, 72, 128])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_many_new_tokens(page, D):
    """512 query rows a sequence or more: keys through LDS."""
    cached_case([130, 140], [130, 400], 16, 2, D, BF16, BF16, page, D + page, extra=8)
    cached_case([129], [1500], 8, 1, D, BF16, BF16, page, D + page + 1, causal=False, in_place=True)
    cached_case([300, 250], [190, 0], 24, 8, D, BF16, BF16, page, D + 2, prefix=page + 9, start=2, behind=5)


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_many_new_tokens_special_values(what):
    def put(k, v):
        v[350, 0, 3], v[351, 0, 9] = what, -what
        v[399] = what
        k[398] = math.nan
    cached_case([140, 130], [400, 500], 16, 1, 64, BF16, BF16, 16, 1, change=put)
    cached_case([140, 130], [400, 500], 16, 1, 128, BF16, BF16, 32, 2, change=put, prefix=70)


@pytest.mark.parametrize("D", [64, 72, 128])
def test_few_tokens_of_many_sequences_behind_a_prefix(D):
    """Many rows over the prefix, few over each sequence's own keys."""
    g = np.random.default_rng(D)
    new = list(g.integers(0, 5, 40))
    cached_case(new, [int(n + x) for n, x in zip(new, g.integers(0, 90, 40))], 16, 2, D, BF16, BF16, 32, D, prefix=700, behind=2)
    cached_case([3] * 60, [3] * 60, 4, 1, D, BF16, BF16, 16, D + 1, prefix=2100, in_place=True, causal=False)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("heads,kv", [(15, 5), (16, 1)])
def test_parts_of_many_rows(heads, kv, dtype, cache):
    """Joined eight rows a workgroup, two of them a wave: of one token, or two."""
    cached_case([150, 0, 140], [1500, 3, 900], heads, kv, 64, dtype, cache, 16, heads, start=1, behind=3)
    cached_case([150, 140], [1200, 700], heads, kv, 32, dtype, cache, 16, heads, prefix=1000)


@pytest.mark.parametrize("heads,kv", [(1, 1), (16, 16), (16, 1), (32, 8), (15, 5), (40, 1), (24, 2)])
def test_cached_head_layouts(heads, kv):
    for dtype, cache in TYPES:
        cached_case([1, 2], [300, 45], heads, kv, 64, dtype, cache, 16, heads + kv)


@pytest.mark.parametrize("dtype,cache", TYPES)
def test_empty_sequences_and_rows_of_none(dtype, cache):
    cached_case([1, 0, 2, 0, 0], [50, 30, 2, 0, 1], 4, 2, 64, dtype, cache, 16, 1, start=2, behind=3)
    cached_case([2, 1], [0, 0], 4, 2, 64, dtype, cache, 16, 2)                # nothing in the cache: zeros
    cached_case([4, 3], [2, 1], 4, 2, 64, dtype, cache, 16, 3)                # more rows than tokens: the first ones see nothing
    cached_case([4, 3], [2, 0], 4, 2, 128, dtype, cache, 16, 4, prefix=40)    # ... but the prefix
    g = np.random.default_rng(7)
    cached_case(list(g.integers(0, 3, 100)), list(g.integers(2, 60, 100)), 2, 1, 64, dtype, cache, 16, 5, behind=1)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("prefix", [1, 16, 100, 1000])
def test_prefixes(prefix, dtype, cache):
    cached_case([1] * 5, [3, 70, 1, 200, 16], 8, 2, 128, dtype, cache, 16, prefix, prefix=prefix)
    cached_case([2, 1, 4], [9, 1, 64], 4, 4, 64, dtype, cache, 64, prefix + 1, prefix=prefix, extra=8, in_place=True)
    cached_case([70, 20], [90, 20], 4, 1, 64, dtype, cache, 32, prefix + 2, prefix=prefix)


@pytest.mark.parametrize("dtype,cache", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_cached_special_values_stay_with_who_sees_them(dtype, cache, what):
    def put(k, v):
        v[27, 0, 3], v[27, 0, 9] = what, -what      # the last but one of the first sequence
        v[28, 0, 5] = what                          # its last token
        k[28, 0] = math.nan
    cached_case([3, 2], [29, 40], 2, 1, 64, dtype, cache, 16, 1, change=put)
    cached_case([20, 2], [29, 40], 2, 1, 128, dtype, cache, 16, 2, change=put)
    cached_case([1, 1], [29, 40], 2, 1, 64, dtype, cache, 16, 3, change=put, prefix=20)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("prefix", [0, 300])
def test_a_query_that_is_nan_over_parts(dtype, cache, prefix):
    """Scores that are all NaN have no largest one; a join of parts answers NaN for them as one part does."""
    g = gen(8)
    lens = [3000, 900, 20]
    pages = Paged(g, lens, 2, 64, cache, 16, prefix)
    fill(pages, g, lens, prefix, dtype)
    p, b = L.make_heads(4, 2, 64, dtype, True), pages.batch([1, 1, 1], lens, prefix)
    q = rand(g, 3, 256).to(dtype)
    n = L.cache_attention_workspace(p, pages.desc, b, 3)
    assert n
    clean, out = (torch.zeros(3, 256, dtype=dtype, device="cuda") for _ in range(2))
    L.laud_cache_attention(p, pages.desc, b, q.cuda(), clean, torch.empty(n, dtype=torch.uint8, device="cuda"))
    q[0, 64:128] = math.nan
    q[2, 70] = math.nan
    L.laud_cache_attention(p, pages.desc, b, q.cuda(), out, torch.empty(n, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    bad = torch.zeros(3, 256, dtype=torch.bool)
    bad[0, 64:128] = bad[2, 64:128] = True
    assert bool(out.cpu()[bad].isnan().all()) and torch.equal(out.cpu()[~bad], clean.cpu()[~bad])


def test_cached_special_values_in_8_bits():
    def put(k, v):
        v[27], v[28] = math.nan, math.inf
        k[28] = math.nan
    cached_case([3, 2], [29, 40], 2, 1, 64, BF16, E4M3, 16, 1, change=put)
    cached_case([20, 2], [29, 40], 2, 1, 128, BF16, E4M3, 16, 2, change=put)


@pytest.mark.parametrize("new", [[1, 2], [90, 40]])
def test_pages_that_are_none_hold_no_keys(new):
    for dtype, cache_type in TYPES:
        g = gen(9)
        lens, n_new = [100, 50], sum(new)
        cache = Paged(g, lens, 2, 64, cache_type, 16)
        fill(cache, g, lens, 0, dtype)
        bad = cache.table.clone()
        bad[0, 2], bad[0, 5], bad[1, 0] = -1, cache.k.shape[0], 2 ** 31 - 1
        gone = [[2, 5], [0]]
        heads = 4 if n_new < 9 else 20
        q = rand(g, n_new, heads * 64).to(dtype)
        out = torch.zeros(n_new, heads * 64, device="cuda", dtype=dtype)
        p = L.make_heads(heads, 2, 64, dtype, True)
        b = L.make_batch(ints(offsets_of(new)), ints(lens), bad)
        ws = torch.empty(max(L.cache_attention_workspace(p, cache.desc, b, n_new), 1), dtype=torch.uint8, device="cuda")
        L.laud_cache_attention(p, cache.desc, b, q.cuda(), out, ws)
        offs = offsets_of(new)
        for i in range(2):
            n, m = lens[i], new[i]
            k, v = (cache.rows64(x, cache.pages[i], n) for x in ("k", "v"))
            allowed = torch.arange(n)[None, :] <= (n - m + torch.arange(m))[:, None]
            for pg in gone[i]:
                allowed[:, 16 * pg:16 * pg + 16] = False
            rows = slice(int(offs[i]), int(offs[i + 1]))
            assert near(out[rows].cpu().view(m, heads, 64), *attend64(q[rows].double().view(m, heads, 64), k, v, p.scale, allowed), n, dtype)


def test_a_long_cache():
    cached_case([1], [20000], 8, 2, 128, BF16, BF16, 16, 1)
    cached_case([1, 1], [9000, 300], 8, 2, 128, BF16, E4M3, 64, 2, prefix=5000)
    cached_case([2], [7000], 4, 1, 64, F32, F32, 128, 3)


# ----- writing and reading -------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cache_type", ["same", E4M3])
@pytest.mark.parametrize("kv,D,page", [(1, 16, 16), (3, 48, 32), (8, 128, 64), (2, 80, 256), (5, 64, 16), (1, 112, 128)])
def test_write_and_read(kv, D, page, cache_type, dtype):
    g = gen(kv + D)
    ct = dtype if cache_type == "same" else E4M3
    lens, new, start, behind = [40, 3, 0, 300, 1, 17], [7, 3, 0, 129, 1, 17], 2, 3
    cache = Paged(g, lens, kv, D, ct, page)
    T = start + sum(new) + behind
    k, v = (rand(g, T, kv * D).to(dtype) * (1e-3 if D == 48 else 1.0) for _ in range(2))
    k[4], v[4] = 0.0, 0.0
    raw = {x: getattr(cache, x).view(torch.uint8).cpu().clone() for x in ("k", "v")}
    b = cache.batch(new, lens, start=start)
    L.laud_cache_write(cache.desc, b, spread(k, 8), spread(v, 16))
    torch.cuda.synchronize()
    offs = offsets_of(new, start)
    touched = torch.zeros(cache.k.shape[0], page, dtype=torch.bool)
    back = {x: spread(torch.full((T, kv * D), 7.0).to(dtype), 24) for x in ("k", "v")}
    L.laud_cache_read(cache.desc, b, back["k"], back["v"])
    for x, rows in (("k", k), ("v", v)):
        held = getattr(cache, x).cpu()
        scales = getattr(cache, x + "s")
        got = back[x].cpu()
        for i, (m, n) in enumerate(zip(new, lens)):
            for r in range(m):
                pos = n - m + r
                pg, at = cache.pages[i][pos // page], pos % page
                touched[pg, at] = True
                row = rows[int(offs[i]) + r].view(kv, D)
                if ct != E4M3:
                    assert torch.equal(held[pg, :, at], row)
                    assert torch.equal(got[int(offs[i]) + r].view(kv, D), row)
                    continue
                f = row.float()
                s = (f.abs().amax(1) / torch.tensor(448.0)).clamp_min(2.0 ** -126)
                assert torch.equal(scales[pg, :, at].cpu(), s)
                codes = (f / s[:, None]).to(E4M3)
                assert torch.equal(held[pg, :, at].float(), codes.float())
                assert torch.equal(got[int(offs[i]) + r].view(kv, D), (codes.float() * s[:, None]).to(dtype))
        # nothing else was written
        mine = touched[:, None, :, None].expand(held.shape)
        elem = held.element_size()
        same = (held.view(torch.uint8) == raw[x]).view(*held.shape, elem).all(-1)
        assert bool(same[~mine].all())
        assert bool((got[:start] == 7).all()) and bool((got[T - behind:] == 7).all())


@pytest.mark.parametrize("cache_type", [BF16, E4M3])
def test_places_that_are_none(cache_type):
    g = gen(3)
    cache = Paged(g, [40, 20], 2, 64, cache_type, 16)
    before = cache.k.view(torch.uint8).clone()
    k, v = (rand(g, 6, 128).to(BF16).cuda() for _ in range(2))
    bad = cache.table.clone()
    bad[0, 2] = cache.k.shape[0]
    bad[1, :] = -7
    for lens in ([40, 20], [1, 2], [10 ** 6, -10], [2 ** 31 - 1, -2 ** 31]):
        b = L.make_batch(ints([0, 3, 6]), ints(lens), bad)
        L.laud_cache_write(cache.desc, b, k, v)
        back = torch.ones(6, 128, device="cuda", dtype=BF16)
        L.laud_cache_read(cache.desc, b, back, back.clone())
        if lens[0] == 1:  # the last of three rows has a place
            assert bool((back[:2] == 0).all()) and bool((back[3:] == 0).all())
            assert torch.equal(back[2], k[2]) or cache_type == E4M3
            cache.k.view(torch.uint8).copy_(before)
        else:
            assert bool((back == 0).all()) and torch.equal(cache.k.view(torch.uint8), before)


def test_quantised_rows_of_special_values():
    cache = Paged(gen(1), [5], 1, 32, E4M3, 16)
    k = rand(gen(2), 5, 32)
    k[1, 3], k[2, 0], k[3] = math.nan, math.inf, 1e-45
    L.laud_cache_write(cache.desc, cache.batch([5], [5]), k.cuda(), k.cuda())
    pg = cache.pages[0][0]
    codes, s = cache.k[pg, 0, :5].float().cpu(), cache.ks[pg, 0, :5].cpu()
    assert bool(codes[1].isnan().all()) and math.isnan(float(s[1]))
    assert bool(codes[2].isnan().any()) and math.isinf(float(s[2]))
    assert float(s[3]) == 2.0 ** -126 and bool((codes[3] == 0).all())
    assert bool(codes[[0, 4]].isfinite().all())


# ----- together -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,cache_type", TYPES)
@pytest.mark.parametrize("prefix", [0, 45])
def test_prompts_and_then_token_by_token(dtype, cache_type, prefix):
    """Prompts are attended to and cached, then answers grow by a token a step, captured and replayed: every row against attention over
    all tokens so far.  Queries, keys and values are columns of one array, as a projection leaves them."""
    g = gen(11 + prefix)
    heads, kv, D, prompt, steps = 6, 2, 64, [37, 1, 0, 140], 6
    widths, B_ = [heads * D, kv * D, kv * D], len(prompt)
    total = [n + steps for n in prompt]
    cache = Paged(g, total, kv, D, cache_type, 16, prefix)
    p = L.make_heads(heads, kv, D, dtype, True)

    def check(got, q, i, seen):
        k, v = (torch.cat((cache.rows64(x, cache.prefix_pages, prefix), cache.rows64(x, cache.pages[i], total[i])[:seen])) for x in ("k", "v"))
        m = got.shape[0]
        allowed = torch.arange(prefix + seen)[None, :] <= (prefix + seen - m + torch.arange(m))[:, None]
        ref = attend64(q.double().view(m, heads, D), k, v, p.scale, allowed)
        assert near(got.view(m, heads, D), *ref, prefix + seen, dtype), (i, seen)

    if prefix:  # the common beginning, over itself and into the cache
        x = rand(g, prefix, sum(widths)).to(dtype)
        q, k, v = x.cuda().split(widths, 1)
        out = torch.zeros(prefix, heads * D, dtype=dtype, device="cuda")
        L.laud_attention(p, ints([0, prefix]), q, k, v, None, out)
        L.laud_cache_write(cache.desc, L.make_batch(ints([0, prefix]), ints([prefix]), ints([cache.prefix_pages])), k, v)
        a, b, c = x.double().split(widths, 1)
        ref = attend64(a.view(-1, heads, D), b.reshape(-1, kv, D), c.reshape(-1, kv, D), p.scale, torch.ones(prefix, prefix).tril().bool())
        assert near(out.cpu().view(-1, heads, D), *ref, prefix, dtype)
    lens = ints(prompt)
    x = rand(g, sum(prompt), sum(widths)).to(dtype)
    q, k, v = x.cuda().split(widths, 1)
    out = torch.zeros(sum(prompt), heads * D, dtype=dtype, device="cuda")
    at = offsets_of(prompt)
    b = L.make_batch(ints(at), lens, cache.table, ints(cache.prefix_pages) if prefix else None, prefix)
    n = L.cache_attention_workspace(p, cache.desc, b, sum(prompt))
    L.laud_cache_write(cache.desc, b, k, v)
    L.laud_cache_attention(p, cache.desc, b, q, out, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    torch.cuda.synchronize()
    for i, n in enumerate(prompt):
        check(out.cpu()[at[i]:at[i + 1]], q.cpu()[at[i]:at[i + 1]], i, n)
    if not prefix and cache_type != E4M3:  # the same rows without a cache
        again = torch.zeros_like(out)
        L.laud_attention(p, ints(at), q, k, v, None, again)
        for i, n in enumerate(prompt):
            check(again.cpu()[at[i]:at[i + 1]], q.cpu()[at[i]:at[i + 1]], i, n)

    new = torch.zeros(B_, sum(widths), dtype=dtype, device="cuda")
    q, k, v = new.split(widths, 1)
    out = torch.zeros(B_, heads * D, dtype=dtype, device="cuda")
    b = L.make_batch(ints(range(B_ + 1)), lens, cache.table, ints(cache.prefix_pages) if prefix else None, prefix)
    n = L.cache_attention_workspace(p, cache.desc, b, B_)
    ws = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")

    def step():
        lens.add_(1)
        L.laud_cache_write(cache.desc, b, k, v)
        L.laud_cache_attention(p, cache.desc, b, q, out, ws)
    graph = None
    for j in range(steps):
        new.copy_(rand(g, B_, sum(widths)).to(dtype))
        if j == 1:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        graph.replay() if graph else step()
        torch.cuda.synchronize()
        for i in range(B_):
            check(out.cpu()[i:i + 1], q.cpu()[i:i + 1], i, prompt[i] + j + 1)
    assert lens.tolist() == total


def test_descriptors_of_another_device():
    cache = Paged(gen(1), [5], 1, 32, BF16, 16)
    b, rows = cache.batch([1], [5]), torch.zeros(1, 32, dtype=BF16, device="cuda")
    p = L.make_heads(1, 1, 32, BF16, True)
    L.laud_cache_write(cache.desc, b, rows, rows)
    for d in (cache.desc, b):
        was, d.device = d.device, 1
        for call in (lambda: L.laud_cache_write(cache.desc, b, rows, rows), lambda: L.laud_cache_read(cache.desc, b, rows, rows.clone()),
                     lambda: L.laud_cache_attention(p, cache.desc, b, rows, rows)):
            with pytest.raises(L.LaudError):
                call()
        d.device = was


# ----- streams and graphs ---------------------------------------------------------------------------------------------------------
def test_run_on_another_stream_and_captured():
    g = gen(4)
    lens, new, prefix = [300, 40, 7], [1, 1, 1], 150
    cache = Paged(g, lens, 2, 64, E4M3, 16, prefix)
    fill(cache, g, lens, prefix, BF16)
    p = L.make_heads(8, 2, 64, BF16, True)
    b = cache.batch(new, lens, prefix)
    q, k, v = (rand(g, 3, c * 64).to(BF16).cuda() for c in (8, 2, 2))
    out = torch.zeros_like(q)
    ws = torch.empty(max(L.cache_attention_workspace(p, cache.desc, b, 3), 1), dtype=torch.uint8, device="cuda")

    def step():
        L.laud_cache_write(cache.desc, b, k, v)
        L.laud_cache_attention(p, cache.desc, b, q, out, ws)
        L.laud_attention(p, b_offsets, out, k, v, None, mixed)
        L.laud_cache_read(cache.desc, b, back[0], back[1])
    b_offsets, mixed, back = ints([0, 1, 3]), torch.zeros_like(q), [torch.zeros_like(k) for _ in range(2)]
    step()
    torch.cuda.synchronize()
    ref = [out.clone(), mixed.clone(), back[0].clone()]
    s = torch.cuda.Stream()
    out.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    assert torch.equal(out, ref[0]) and torch.equal(mixed, ref[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        out.fill_(1.0)
        ws.fill_(i)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(mixed, ref[1]) and torch.equal(back[0], ref[2])
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, ref[0])


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new", [1, 150])
def test_a_cache_of_more_than_32_bits(new, dtype, cache):
    """Pages whose first element lies beyond 2^32 elements, and some that do not."""
    kv, D, page, heads = 8, 128, 256, 32
    pages = (1 << 32) // (kv * D * page) + 40
    kc, vc = (torch.empty(pages, kv, page, D, dtype=torch.uint8 if cache == E4M3 else cache, device="cuda") for _ in range(2))
    scales = [torch.empty(pages, kv, page, device="cuda") for _ in range(2)] if cache == E4M3 else [None, None]
    if cache == E4M3:
        kc, vc = kc.view(E4M3), vc.view(E4M3)
    desc = L.make_cache(kc, vc, *scales)
    g = gen(new)
    lens, table = [700, new], [[pages - 1, 3, pages - 17], [pages - 30, -1, -1]]
    k, v = (rand(g, sum(lens), kv * D).to(dtype) for _ in range(2))
    every = L.make_batch(ints(offsets_of(lens)), ints(lens), ints(table))
    L.laud_cache_write(desc, every, k.cuda(), v.cuda())
    kb, vb = (torch.zeros_like(k, device="cuda") for _ in range(2))
    L.laud_cache_read(desc, every, kb, vb)
    b = L.make_batch(ints(offsets_of([new, new])), ints(lens), ints(table))
    p = L.make_heads(heads, kv, D, dtype, True)
    q = rand(g, 2 * new, heads * D).to(dtype)
    out = torch.zeros(2 * new, heads * D, dtype=dtype, device="cuda")
    n = L.cache_attention_workspace(p, desc, b, 2 * new)
    L.laud_cache_attention(p, desc, b, q.cuda(), out, torch.empty(max(n, 1), dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    if cache != E4M3:
        assert torch.equal(kb.cpu(), k) and torch.equal(vb.cpu(), v)
    for i, (j, m) in enumerate(zip(offsets_of(lens), lens)):
        rows = []
        for held, s in zip((kc, vc), scales):
            x = held.view(torch.uint8)[table[i]].view(cache).float().cpu().double()
            x = x if s is None else x * s[table[i]].cpu().double()[..., None]
            rows.append(x.permute(0, 2, 1, 3).reshape(-1, kv, D)[:m])
        allowed = torch.arange(m)[None, :] <= (m - new + torch.arange(new))[:, None]
        ref = attend64(q[i * new:(i + 1) * new].double().view(new, heads, D), *rows, p.scale, allowed)
        assert near(out.cpu()[i * new:(i + 1) * new].view(new, heads, D), *ref, m, dtype)


def test_the_same_call_gives_the_same_bits():
    g = gen(5)
    q, k, v = (rand(g, 700, c * 64).to(BF16).cuda() for c in (4, 2, 2))
    p, offs = L.make_heads(4, 2, 64, BF16, True), ints([0, 333, 700])
    outs = [torch.zeros_like(q) for _ in range(3)]
    for o in outs:
        L.laud_attention(p, offs, q, k, v, None, o)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
