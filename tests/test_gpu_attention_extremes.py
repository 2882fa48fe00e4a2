"""Scores at the ends of float32, through every kernel: as rows of a call (few of them, and tiles), over a cache (one part, several joined, tiles).

Where all scores are the same number all weights are the same, and a result is the mean of the values that its query sees: a sum of n values in
float32, off by at most n 2^-24 of the sum of magnitudes, the division 2^-23, the rounding of the result, and that of a weight where it meets
bf16 values (2^-8 in tiles, 2^-15 elsewhere; a weight of 1 is not rounded, but in 8 bits its product with the value's scale is).  The tokens whose score is far above all others have all of the
weight, 1 each, and the result is their values' mean."""
import math

import pytest
import torch

import paper_2308_15949_amd as L
from test_gpu_attention import BF16, E4M3, F32, HALF, Paged, gen, ints, rand, spread

pytestmark = pytest.mark.gpu

# form: kind, query heads of one key head, new tokens, tokens
FORMS = {"few": ("rows", 2, 150, 150), "tiles": ("rows", 192, 150, 150), "kept": ("kept", 192, 150, 150), "few_kept": ("kept", 2, 150, 150),
         "cache": ("cache", 4, 3, 200), "rows_of_a_cache": ("cache", 4, 20, 200), "joined": ("cache", 2, 3, 3000), "joined_rows": ("cache", 2, 40, 3000),
         "joined_many": ("cache", 16, 300, 1400), "tiles_of_a_cache": ("cache", 16, 140, 200)}
TYPES = [(BF16, BF16), (BF16, E4M3), (F32, F32)]


def cases(*left_out):
    return [pytest.param(form, *t, id=f"{form}-{str(t[0])[6:]}-{str(t[1])[6:]}") for form, f in FORMS.items() for t in TYPES
            if form not in left_out and (f[0] == "cache" or t[0] == t[1])]


def attend(form, dtype, cache_type, q, k, v, scale, D=64, value_scales={}):
    """q, k, v [tokens][D]: every query head has the same q.  Result [new][heads][D], the values as they are held [tokens][D].  value_scales: of
    tokens whose scale in an 8-bit cache is replaced."""
    kind, heads, new, tokens = FORMS[form]
    rows = q[tokens - new:].to(dtype)[:, None, :].expand(new, heads, D).reshape(new, heads * D)
    qd, kd, vd = spread(rows, 8), k.to(dtype).cuda(), v.to(dtype).cuda()
    out = torch.full_like(qd, 7.0)
    p = L.make_heads(heads, 1, D, dtype, True, scale)
    if kind != "cache":
        keep = torch.ones(tokens, dtype=torch.uint8, device="cuda") if kind == "kept" else None
        L.laud_attention(p, ints([0, tokens]), qd, kd, vd, keep, out)
        held = v.to(dtype).double()
    else:
        cache = Paged(gen(1), [tokens], 1, D, cache_type, 16)
        L.laud_cache_write(cache.desc, cache.batch([tokens], [tokens]), kd, vd)
        for t, x in value_scales.items():
            cache.vs[cache.pages[0][t // 16], 0, t % 16] = x
        b = cache.batch([new], [tokens])
        n = L.cache_attention_workspace(p, cache.desc, b, new)
        assert (n > 0) == form.startswith("joined")
        L.laud_cache_attention(p, cache.desc, b, qd, out, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
        held = cache.rows64("v", cache.pages[0], tokens)[:, 0]
    torch.cuda.synchronize()
    return out.cpu().double().view(new, heads, D), held


def means(form, held, first=0):
    """Of the values from `first` on that each query sees, and of their magnitudes."""
    _, _, new, tokens = FORMS[form]
    n = torch.arange(tokens - new + 1, tokens + 1, dtype=torch.float64)[:, None] - first
    return ((x[first:].cumsum(0)[tokens - new - first:] / n)[:, None, :] for x in (held, held.abs()))


def near_mean(form, got, held, dtype, cache_type, first=0):
    ref, size = means(form, held, first)
    tiled = "tiles" in form or form in ("kept", "joined_many")
    weight = 0.0 if dtype == F32 else 2.0 ** -8 if tiled and cache_type == BF16 else 2.0 ** -15
    return bool(((got - ref).abs() <= HALF[dtype] * ref.abs() + size * (len(held) * 2.0 ** -24 + 2.0 ** -20 + weight)).all())


# 63 equal products whose sum is close to 2^e, a sixteenth of that for a score; times log2(e) it is no number of float32.
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("e", [0, 26, 31, 40, 80, 126])
@pytest.mark.parametrize("form,dtype,cache_type", cases())
def test_equal_scores_of_any_size(form, dtype, cache_type, e, sign):
    tokens = FORMS[form][3]
    q = torch.full((tokens, 64), 2.0 ** ((e - 6) // 2))
    k = torch.full((tokens, 64), sign * 2.0 ** ((e - 6) - (e - 6) // 2))
    q[:, 0] = 0.0
    if cache_type == E4M3:  # (a scale that is a power of two, so that codes and scores are what they are in bf16)
        k[:, 0] = k[:, 0] * 1.75
    v = rand(gen(e), tokens, 64)
    got, held = attend(form, dtype, cache_type, q, k, v, 0.0625)
    assert near_mean(form, got, held, dtype, cache_type)


@pytest.mark.parametrize("form,dtype,cache_type", cases())
def test_one_score_far_above_the_others(form, dtype, cache_type):
    """Scores grow to the last token, or fall from the first one, by steps far above any exponent's range."""
    tokens = FORMS[form][3]
    at = torch.arange(tokens, dtype=torch.float32)
    v = rand(gen(3), tokens, 64)
    for grow in (True, False):
        k = ((at if grow else tokens - at) // 8 * 2.0 ** 40)[:, None].expand(tokens, 64)  # (numbers of bf16; eight alike)
        got, held = attend(form, dtype, cache_type, torch.full((tokens, 64), 2.0), k, v, 0.125)
        new = FORMS[form][2]
        kk = k[:, 0].to(dtype).float()
        for i in range(new):
            seen = tokens - new + i + 1
            best = (kk[:seen] == kk[:seen].max()).nonzero()[:, 0]
            x = held[best]
            ref, size = x.mean(0), x.abs().mean(0)
            assert bool(((got[i] - ref).abs() <= HALF[dtype] * ref.abs() + size * (len(best) * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -15 if cache_type == E4M3 else 0))).all()), (grow, i)


def hopeless(form):
    """Tokens whose score is -infinity: a beginning that fills parts, and some near the end, where queries see different numbers of them."""
    tokens = FORMS[form][3]
    return [*range(400 if tokens > 1000 else 40), tokens - 90, tokens - 89, tokens - 40, tokens - 7, tokens - 2]


def check_hopeless(form, dtype, cache_type, got, held):
    """Rows without a weight are zeros, others the mean of the values with one, but for elements of values that are not finite: these are not
    finite where the query sees them."""
    _, heads, new, tokens = FORMS[form]
    weight = torch.ones(tokens, 1, dtype=torch.float64)
    weight[hopeless(form)] = 0
    bad = ~held.isfinite()
    x = torch.where(bad, 0.0, held) * weight
    first = tokens - new
    n = weight.cumsum(0)[first:]
    ref, size = ((y.cumsum(0)[first:] / n.clamp_min(1))[:, None, :].expand(new, heads, 64) for y in (x, x.abs()))
    spoilt = ((bad.cumsum(0) > 0)[first:] & (n > 0))[:, None, :].expand(new, heads, 64)
    assert not bool(got[spoilt].isfinite().any())
    tol = HALF[dtype] * ref.abs() + size * (tokens * 2.0 ** -24 + 2.0 ** -20 + (2.0 ** -15 if cache_type == E4M3 else 0.0))
    assert bool(((got - ref).abs() <= tol)[~spoilt].all())
    none = (n == 0)[:, 0]
    assert bool((got[none] == 0).all()) and bool(none.any()) == (new == tokens)


def hopeless_case(form, dtype, cache_type, change, **more):
    tokens = FORMS[form][3]
    k, v = torch.zeros(tokens, 64), rand(gen(5), tokens, 64)
    k[hopeless(form)] = -3.0e38
    change(v)
    check_hopeless(form, dtype, cache_type, *attend(form, dtype, cache_type, torch.ones(tokens, 64), k, v, 1.0, **more))


@pytest.mark.parametrize("form,dtype,cache_type", cases())
def test_scores_of_minus_infinity_have_no_weight(form, dtype, cache_type):
    hopeless_case(form, dtype, cache_type, lambda v: None)


@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("form,dtype,cache_type", cases())
def test_values_that_are_not_finite_show_whatever_their_weight(form, dtype, cache_type, what):
    tokens = FORMS[form][3]

    def put(v):  # (in steps that all queries see, and in such as some do not)
        v[5, 3] = v[39, 63] = v[tokens - 90, 20] = v[tokens - 40, 21] = what
        v[tokens - 7, 9], v[tokens - 2, 11] = what, -what
    hopeless_case(form, dtype, cache_type, put)

    def near_the_end(v):  # (an 8-bit row is NaN as a whole: some queries do not see this one)
        v[tokens - 2, 30] = what
    hopeless_case(form, dtype, cache_type, near_the_end)

    def with_a_weight(v):
        v[tokens - 3, 1], v[tokens - 80, 2] = what, -what
    hopeless_case(form, dtype, cache_type, with_a_weight)


@pytest.mark.parametrize("what", [math.nan, math.inf])
@pytest.mark.parametrize("where", ["beginning", "end", "weight"])
@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][0] == "cache"])
def test_scales_that_are_not_finite_show_whatever_their_weight(form, where, what):
    t = FORMS[form][3] - 2 if where == "end" else FORMS[form][3] - 3 if where == "weight" else 17
    hopeless_case(form, BF16, E4M3, lambda v: None, value_scales={t: what})
