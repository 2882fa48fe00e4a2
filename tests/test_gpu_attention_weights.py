"""Bits of the softmax' weights where few rows meet values in bf16 or 8 bits: two parts, cut off behind eight bits and rounded by half a step
(2^-8) of the 2^-7 that are left, 2^-15 together.  The other terms of the tolerance are those of test_gpu_attention.py."""
import pytest
import torch

import paper_2308_15949_amd as L
from test_gpu_attention import BF16, E4M3, HALF, Paged, attend64, fill, gen, ints, offsets_of, rand

pytestmark = pytest.mark.gpu


def close(got, ref, size, off, n):
    got = got.double().cpu()
    tol = HALF[BF16] * ref.abs() + size * (2 * off + n * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -15)
    return bool(((got - ref).abs() <= tol).all())


@pytest.mark.parametrize("new,heads,kv,D,causal,share", [
    ([300, 5], 8, 2, 64, True, 1.0), ([700], 4, 4, 128, False, 1.0), ([150, 33], 16, 1, 80, True, 0.6), ([8] * 60, 20, 5, 128, False, 1.0),
    ([5, 8, 1, 0, 7] * 30, 16, 16, 64, True, 0.8), ([13, 14, 20, 9] * 20, 32, 8, 96, True, 1.0)])
def test_few_rows_and_short_sequences(new, heads, kv, D, causal, share):
    g = gen(heads + D)
    T = sum(new)
    q, k, v = (rand(g, T, h * D).to(BF16) for h in (heads, kv, kv))
    keep = torch.rand(T, generator=g) < share
    p = L.make_heads(heads, kv, D, BF16, causal)
    out = torch.zeros_like(q, device="cuda")
    L.laud_attention(p, ints(offsets_of(new)), q.cuda(), k.cuda(), v.cuda(), keep.to(torch.uint8).cuda() if share < 1 else None, out)
    torch.cuda.synchronize()
    offs = offsets_of(new)
    for i, j in zip(offs, offs[1:]):
        n = int(j - i)
        allowed = keep[i:j, None] & keep[None, i:j]
        allowed = allowed.tril() if causal else allowed
        ref = attend64(q[i:j].double().view(n, heads, D), k[i:j].double().view(n, kv, D), v[i:j].double().view(n, kv, D), p.scale, allowed)
        assert close(out[i:j].view(n, heads, D), *ref, n), (i, j)


@pytest.mark.parametrize("cache_type", [BF16, E4M3])
@pytest.mark.parametrize("new,lens,heads,kv,D,prefix", [
    ([1, 1], [2000, 70], 8, 2, 128, 0), ([1, 3, 2], [500, 40, 33], 6, 3, 80, 0), ([9, 30], [300, 200], 8, 2, 64, 0),
    ([1] * 20, list(range(1, 400, 20)), 8, 2, 128, 700), ([40, 40], [90, 60], 4, 1, 64, 150)])
def test_over_a_cache(new, lens, heads, kv, D, prefix, cache_type):
    g = gen(D + prefix)
    cache = Paged(g, lens, kv, D, cache_type, 16, prefix)
    fill(cache, g, lens, prefix, BF16)
    T = sum(new)
    q = rand(g, T, heads * D).to(BF16)
    out = torch.zeros_like(q, device="cuda")
    p, b = L.make_heads(heads, kv, D, BF16, True), cache.batch(new, lens, prefix)
    n = L.cache_attention_workspace(p, cache.desc, b, T)
    L.laud_cache_attention(p, cache.desc, b, q.cuda(), out, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
    torch.cuda.synchronize()
    kp, vp = (cache.rows64(x, cache.prefix_pages, prefix) for x in ("k", "v"))
    offs = offsets_of(new)
    for i, (m, pages, ln) in enumerate(zip(new, cache.pages, lens)):
        k, v = (torch.cat((a, cache.rows64(x, pages, ln))) for x, a in (("k", kp), ("v", vp)))
        allowed = torch.arange(prefix + ln)[None, :] <= (prefix + ln - m + torch.arange(m))[:, None]
        rows = slice(int(offs[i]), int(offs[i + 1]))
        assert close(out[rows].view(m, heads, D), *attend64(q[rows].double().view(m, heads, D), k, v, p.scale, allowed), prefix + ln), i
