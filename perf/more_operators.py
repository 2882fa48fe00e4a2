"""Workloads of the attention of a token block: over the tokens of packed sequences, and of new tokens over a paged cache of keys and
values, which is written, quantised on the way where it is held in 8 bits, read back, and may begin with pages that a batch shares.

A case is a dict of plain values.  listed() names the standing ones, draw() gives more of the same ranges, prepare() makes what a
program has in hand before the call, run() is one pass through an operator: in its plain form, elementary operations in 32 bits
(own = False), or through this package's entry points (own = True).  work() is what a pass cannot do without, exact() the result
in 64 bits from the definition.

Definitions
  attention  out[t, h] = sum_j w_j v[j, h / G],  w = softmax_j(scale q[t, h] . k[j, h / G]) over the tokens j of t's sequence, up to
             t itself where it is causal; a token whose keep is 0 is neither a query (its row is zeros) nor a key
  write      new token i of sequence b, of n_b new ones, goes to position len_b - n_b + i: page table[b, position / page], row
             position % page; in 8 bits a scale a token and head: s = max(max|x| / 448, 2^-126), codes e4m3(x / s)
  read       the rows at those positions, code * s
  cached     out as above for new tokens over the cached ones of their sequence up to themselves, behind the tokens of a prefix
             that all sequences share
8-bit results are returned as float8 tensors (the values of the codes) beside their scales.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
E4M3 = torch.float8_e4m3fn


# ----- cases ------------------------------------------------------------------------------------------------------------
# seqs sequences; `mix` seeds how their lengths (new: tokens of this call, past: tokens in the cache before it) are spread below the
# given largest ones, 0: all are the largest
def listed() -> list[dict]:
    return [
        # image tokens (14 x 14 and one more) of five samples in float32
        dict(name="attend_images_f32", op="attend", seqs=5, new=197, mix=0, heads=16, kv_heads=16, D=64, dtype="f32", causal=False,
             keep=1.0),
        # tokens that a masker thinned out, a head width between the powers of two
        dict(name="attend_kept_tokens", op="attend", seqs=3, new=577, mix=0, heads=12, kv_heads=12, D=80, dtype="bf16", causal=False,
             keep=0.66),
        # prompts of different lengths packed one behind the other, four query heads to a key head
        dict(name="attend_packed_prompts", op="attend", seqs=12, new=2000, mix=5, heads=32, kv_heads=8, D=128, dtype="bf16", causal=True,
             keep=1.0),
        # one long document
        dict(name="attend_long_prompt", op="attend", seqs=1, new=16384, mix=0, heads=16, kv_heads=4, D=128, dtype="bf16", causal=True,
             keep=1.0),
        # the step of a decoder on four sequences: what one token adds to the cache
        dict(name="write_step", op="write", seqs=4, new=1, past=300, mix=1, kv_heads=8, D=128, dtype="bf16", cache="bf16", page=16),
        # prompts written in 8 bits
        dict(name="write_prompts_e4m3", op="write", seqs=12, new=2000, past=100, mix=2, kv_heads=8, D=128, dtype="bf16", cache="e4m3",
             page=64),
        # the cache of a small float32 model read back, a width that is no power of two
        dict(name="read_f32", op="read", seqs=5, new=197, past=0, mix=3, kv_heads=12, D=80, dtype="f32", cache="f32", page=16),
        # 8-bit prompts read back for another pass
        dict(name="read_prompts_e4m3", op="read", seqs=12, new=2000, past=0, mix=4, kv_heads=8, D=128, dtype="bf16", cache="e4m3",
             page=64),
        # one conversation far into its length: a row of queries against a long cache
        dict(name="step_one_long", op="cached", seqs=1, new=1, past=32767, mix=0, heads=32, kv_heads=8, D=128, dtype="bf16", cache="bf16",
             page=16, prefix=0),
        # a server's step: sequences of all lengths, cache in 8 bits
        dict(name="step_batch_e4m3", op="cached", seqs=64, new=1, past=8000, mix=6, heads=32, kv_heads=8, D=128, dtype="bf16",
             cache="e4m3", page=64, prefix=0),
        # a few drafted tokens of a small float32 model behind shared instructions
        dict(name="prefix_small_f32", op="cached", seqs=3, new=5, past=60, mix=7, heads=8, kv_heads=4, D=64, dtype="f32", cache="f32",
             page=16, prefix=1000),
        # a batch of answers to one long document
        dict(name="prefix_batch", op="cached", seqs=32, new=1, past=500, mix=8, heads=32, kv_heads=8, D=128, dtype="bf16", cache="bf16",
             page=64, prefix=16384),
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng) -> dict:
    op = rng.choice(("attend", "attend", "write", "read", "cached", "cached", "cached"))
    while True:
        group, kv, D = rng.choice((1, 1, 2, 4, 5, 8)), rng.choice((1, 2, 4, 8, 12, 16)), rng.choice((32, 64, 64, 80, 96, 128, 128, 128))
        dtype, mix = rng.choice(("bf16", "bf16", "f32")), rng.randint(1, 10 ** 6)
        c = dict(op=op, heads=group * kv, kv_heads=kv, D=D, dtype=dtype, mix=mix)
        if group * kv > 40:
            continue
        if op == "attend":
            c.update(seqs=_log_int(rng, 1, 64), new=_log_int(rng, 1, 8192), causal=rng.random() < 0.6,
                     keep=rng.choice((1.0, 1.0, round(rng.uniform(0.0, 0.95), 2))))
            limit = 1.0e12 if dtype == "bf16" else 1.0e11
        else:
            cache = rng.choice((dtype, "e4m3")) if dtype == "bf16" or op != "cached" else dtype
            c.update(cache=cache, page=rng.choice((16, 32, 64, 128)))
            if op == "cached":
                c.update(seqs=_log_int(rng, 1, 64), new=rng.choice((1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 600))),
                         past=_log_int(rng, 1, 32768) - 1, prefix=rng.choice((0, 0, _log_int(rng, 16, 16384))))
                limit = 4.0e11 if dtype == "bf16" else 4.0e10
            else:
                del c["heads"]
                c.update(seqs=_log_int(rng, 1, 64), new=_log_int(rng, 1, 4096), past=rng.choice((0, _log_int(rng, 1, 2000))))
                limit = 0.0
        w = work(c)
        if w["bytes"] <= 6.0e8 and (not limit or w["flops"] <= limit):
            return c


def _sizes(case: dict) -> tuple[list[int], list[int]]:
    """The sequences' new tokens, and all their tokens in the cache behind this call."""
    rng = random.Random(case["mix"])

    def spread(most: int, least: int) -> list[int]:
        if not case["mix"] or most <= least + 1:
            return [most] * case["seqs"]
        return [rng.randint(least, most) if rng.random() < 0.8 else rng.randint(least, max(least, most // 8)) for _ in range(case["seqs"])]

    # (prompts of one token occur; a batch's new tokens are one each, or as many as were drafted)
    new = spread(case["new"], 1)
    past = spread(case.get("past", 0), 0)
    return new, [n + p for n, p in zip(new, past)]


# ----- inputs -----------------------------------------------------------------------------------------------------------
class _Rand:
    def __init__(self, seed: int):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV)

    def heads(self, n: int, heads: int, D: int, dtype):
        """Rows of a projection's result: channels of different size."""
        size = torch.exp(0.3 * self.normal(heads * D))
        return (self.normal(n, heads * D) * size).to(dtype)

    def order(self, n: int):
        return torch.randperm(n, generator=self.g, device=DEV).to(torch.int32)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _offsets(lens: list[int]) -> list[int]:
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _pages(n: int, page: int) -> int:
    return -(-n // page)


def prepare(case: dict, seed: int) -> dict:
    r = _Rand(seed)
    new, lens = _sizes(case)
    H, D, dt, T = case["kv_heads"], case["D"], TYPES[case["dtype"]], sum(new)
    s = {"case": case, "new": new, "lens": lens, "at": _offsets(new), "offsets": _ints(_offsets(new)), "scale": 1.0 / math.sqrt(D)}
    if case["op"] == "attend":
        # the three parts of one projection's result, side by side in its rows
        C, Ck = case["heads"] * D, H * D
        rows = torch.cat((r.heads(T, case["heads"], D, dt), r.heads(T, H, D, dt), r.heads(T, H, D, dt)), 1)
        s["q"], s["k"], s["v"] = rows[:, :C], rows[:, C:C + Ck], rows[:, C + Ck:]
        s["keep"] = None if case["keep"] >= 1.0 else (r.uniform(T) < case["keep"]).to(torch.uint8)
        s["out"] = torch.empty(T, C, device=DEV, dtype=dt)
        return s
    page, ct = case["page"], TYPES[case["cache"]]
    shared = _pages(case.get("prefix", 0), page)
    need = [_pages(n, page) for n in lens]
    pages = shared + sum(need) + 3
    # a cache that has been in use: every row holds keys and values, pages belong to sequences in no order
    for n in ("k", "v"):
        x = r.normal(pages, H, page, D) * torch.exp(0.3 * r.normal(H, 1, D))
        s[n + "_scale"] = None
        if case["cache"] == "e4m3":
            scale = (x.abs().amax(-1) / torch.tensor(448.0, device=DEV)).clamp_min(2.0 ** -126)
            x, s[n + "_scale"] = x / scale[..., None], scale
        s[n + "_cache"] = x.to(ct)
    order = r.order(pages)
    s["prefix"] = order[:shared].clone() if shared else None
    table = torch.full((len(lens), max(need) + 1), -1, dtype=torch.int32, device=DEV)
    at = shared
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    s["table"], s["lens_dev"] = table, _ints(lens)
    if case["op"] == "cached":
        s["q"] = r.heads(T, case["heads"], D, dt)
        s["out"] = torch.empty_like(s["q"])
    elif case["op"] == "write":
        s["k"], s["v"] = r.heads(T, H, D, dt), r.heads(T, H, D, dt)
    else:
        s["k"], s["v"] = (torch.empty(T, H * D, device=DEV, dtype=dt) for _ in range(2))
    return s


# ----- one pass ---------------------------------------------------------------------------------------------------------
def run(state: dict):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _softmax_rows(logits):
    """Weights over the last axis; a row without a finite logit gets zeros."""
    top = logits.amax(-1, keepdim=True)
    w = torch.exp(logits - torch.where(torch.isinf(top), 0.0, top))
    return w / w.sum(-1, keepdim=True).clamp_min(1e-30)


def _attend32(q, k, v, scale: float, first, allowed=None):
    """q [n][heads][D] over k, v [m][kv][D], in 32 bits.  first: keys that the first query sees besides itself, each further query one
    more (None: all see all); allowed: truth values of the keys."""
    n, heads, D = q.shape
    m, kv, _ = k.shape
    group = heads // kv
    out = torch.empty(n, kv, group, D, device=q.device)
    rows = q.float().view(n, kv, group, D).transpose(0, 1).contiguous()
    kt, vt = k.float().permute(1, 2, 0).contiguous(), v.float().transpose(0, 1).contiguous()
    at = torch.arange(m, device=q.device)
    part = max(1, (1 << 28) // max(1, m * heads))
    for i in range(0, n, part):
        j = min(n, i + part)
        logits = torch.bmm(rows[:, i:j].reshape(kv, -1, D), kt).view(kv, j - i, group, m) * scale
        if first is not None:
            seen = at[None, :] <= first + torch.arange(i, j, device=q.device)[:, None]
            logits = logits.masked_fill(~seen[:, None, :], -math.inf)
        if allowed is not None:
            logits = logits.masked_fill(~allowed, -math.inf)
        w = _softmax_rows(logits).view(kv, -1, m)
        out[i:j] = torch.bmm(w, vt).view(kv, j - i, group, D).transpose(0, 1)
    return out.view(n, heads, D)


def _plain_attend(s):
    c = s["case"]
    T, H, Hk, D = len(s["out"]), c["heads"], c["kv_heads"], c["D"]
    q, k, v = s["q"].reshape(T, H, D), s["k"].reshape(T, Hk, D), s["v"].reshape(T, Hk, D)
    kept = None if s["keep"] is None else s["keep"] != 0
    for i, j in zip(s["at"], s["at"][1:]):
        out = _attend32(q[i:j], k[i:j], v[i:j], s["scale"], 0 if c["causal"] else None, None if kept is None else kept[i:j])
        if kept is not None:
            out = torch.where(kept[i:j, None, None], out, 0.0)
        s["out"][i:j] = out.view(j - i, H * D).to(s["out"].dtype)
    return s["out"]


def _raw(cache):
    return cache.view(torch.uint8) if cache.dtype == E4M3 else cache


def _places(s):
    """Page and row of every new token's place in the cache."""
    c = s["case"]
    pages, rows = [], []
    for b, (n, m) in enumerate(zip(s["new"], s["lens"])):
        at = torch.arange(m - n, m, device=DEV)
        pages.append(s["table"][b].long()[at // c["page"]])
        rows.append(at % c["page"])
    return torch.cat(pages), torch.cat(rows)


def _cached_rows(s, n: str, pages, rows):
    """[tokens][kv][D] in 32 bits."""
    x = _raw(s[n + "_cache"])[pages, :, rows]
    if s[n + "_scale"] is None:
        return x.float()
    return x.view(E4M3).float() * s[n + "_scale"][pages, :, rows][..., None]


def _plain_write(s):
    c = s["case"]
    pages, rows = _places(s)
    got = {}
    for n in ("k", "v"):
        x = s[n].view(-1, c["kv_heads"], c["D"])
        if c["cache"] == "e4m3":
            x = x.float()
            scale = (x.abs().amax(-1) / torch.tensor(448.0, device=DEV)).clamp_min(2.0 ** -126)
            s[n + "_scale"][pages, :, rows] = scale
            x = (x / scale[..., None]).to(E4M3).view(torch.uint8)
            got[n + "_scale"] = s[n + "_scale"]
        _raw(s[n + "_cache"])[pages, :, rows] = x
        got[n] = s[n + "_cache"]
    return got


def _plain_read(s):
    pages, rows = _places(s)
    for n in ("k", "v"):
        s[n].copy_(_cached_rows(s, n, pages, rows).view(s[n].shape))
    return {"k": s["k"], "v": s["v"]}


def _plain_cached(s):
    c = s["case"]
    H, D, page, shared = c["heads"], c["D"], c["page"], c["prefix"]
    q = s["q"].view(-1, H, D)
    before = torch.arange(shared, device=DEV)
    for b, (n, m) in enumerate(zip(s["new"], s["lens"])):
        at = torch.arange(m, device=DEV)
        pages, rows = s["table"][b].long()[at // page], at % page
        if shared:
            pages, rows = torch.cat((s["prefix"].long()[before // page], pages)), torch.cat((before % page, rows))
        i = s["at"][b]
        out = _attend32(q[i:i + n], _cached_rows(s, "k", pages, rows), _cached_rows(s, "v", pages, rows), s["scale"], shared + m - n)
        s["out"][i:i + n] = out.view(n, H * D).to(s["out"].dtype)
    return s["out"]


_PLAIN = {"attend": _plain_attend, "write": _plain_write, "read": _plain_read, "cached": _plain_cached}


def _own_attend(s):
    from paper_2308_15949_amd import binding as B
    c = s["case"]
    if "p" not in s:
        s["p"] = B.make_heads(c["heads"], c["kv_heads"], c["D"], s["q"].dtype, c["causal"], s["scale"])
    B.laud_attention(s["p"], s["offsets"], s["q"], s["k"], s["v"], s["keep"], s["out"])
    return s["out"]


def _own_cache(s):
    from paper_2308_15949_amd import binding as B
    if "cache" not in s:
        s["cache"] = B.make_cache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        s["batch"] = B.make_batch(s["offsets"], s["lens_dev"], s["table"], s["prefix"], s["case"].get("prefix", 0))
    return s["cache"], s["batch"]


def _own_write(s):
    from paper_2308_15949_amd import binding as B
    B.laud_cache_write(*_own_cache(s), s["k"], s["v"])
    got = {"k": s["k_cache"], "v": s["v_cache"]}
    if s["k_scale"] is not None:
        got["k_scale"], got["v_scale"] = s["k_scale"], s["v_scale"]
    return got


def _own_read(s):
    from paper_2308_15949_amd import binding as B
    B.laud_cache_read(*_own_cache(s), s["k"], s["v"])
    return {"k": s["k"], "v": s["v"]}


def _own_cached(s):
    from paper_2308_15949_amd import binding as B
    c = s["case"]
    cache, batch = _own_cache(s)
    if "p" not in s:
        s["p"] = B.make_heads(c["heads"], c["kv_heads"], c["D"], s["q"].dtype, True, s["scale"])
        n = B.cache_attention_workspace(s["p"], cache, batch, len(s["q"]))
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    B.laud_cache_attention(s["p"], cache, batch, s["q"], s["out"], s["ws"])
    return s["out"]


_OWN = {"attend": _own_attend, "write": _own_write, "read": _own_read, "cached": _own_cached}


# ----- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case: dict) -> dict:
    new, lens = _sizes(case)
    T, D, Hk = sum(new), case["D"], case["kv_heads"]
    e = BYTES[case["dtype"]]
    if case["op"] == "attend":
        H, kept = case["heads"], case["keep"]
        pairs = sum(n * (n + 1) / 2 if case["causal"] else n * n for n in new) * kept * kept
        # (a skipped token's q, k and v are not needed, its row of zeros is written)
        nbytes = T * D * e * (H + kept * (H + 2 * Hk)) + 4 * len(new) + (T if kept < 1.0 else 0)
        return {"bytes": nbytes, "flops": 4 * D * H * pairs}
    held = Hk * (D * BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0))  # bytes of a token's keys, or values
    if case["op"] in ("write", "read"):
        return {"bytes": 2 * T * (Hk * D * e + held) + 12 * len(new), "flops": 6 * T * Hk * D if case["cache"] == "e4m3" else 0}
    H, shared = case["heads"], case["prefix"]
    pairs = sum(n * (shared + m - n) + n * (n + 1) / 2 for n, m in zip(new, lens))
    return {"bytes": 2 * held * (shared + sum(lens)) + 2 * T * H * D * e, "flops": 4 * D * H * pairs}


# ----- the result in 64 bits, from the definitions --------------------------------------------------------------------------
def exact(case: dict, seed: int):
    s = prepare(case, seed)
    H, D = case["kv_heads"], case["D"]
    starts = [0]
    for n in s["new"]:
        starts.append(starts[-1] + n)

    def place(table_row, i: int):
        return int(table_row[i // case["page"]]), i % case["page"]

    if case["op"] in ("write", "read"):
        tables = s["table"].tolist()
        where = [place(tables[b], m - n + i) for b, (n, m) in enumerate(zip(s["new"], s["lens"])) for i in range(n)]
        at = torch.tensor(where, device=DEV).t().contiguous()
        slot = at[0] * case["page"] + at[1]  # of the cache with its pages one behind the other
        got = {}
        for n in ("k", "v"):
            held = s[n + "_cache"].double().permute(0, 2, 1, 3).reshape(-1, H, D)
            scale = None if s[n + "_scale"] is None else s[n + "_scale"].double().permute(0, 2, 1).reshape(-1, H)
            if case["op"] == "read":
                x = held[slot] if scale is None else held[slot] * scale[slot].unsqueeze(2)
                got[n] = x.reshape(len(where), H * D)
                continue
            x = s[n].double().reshape(len(where), H, D)
            shape = s[n + "_cache"].shape
            if scale is not None:
                each = (x.abs().max(2).values / 448.0).float().double().clamp(min=2.0 ** -126)
                x = (x / each.unsqueeze(2)).to(E4M3).double()
                scale[slot] = each
                got[n + "_scale"] = scale.reshape(shape[0], shape[2], H).transpose(1, 2).contiguous()
            held[slot] = x
            got[n] = held.reshape(shape[0], shape[2], H, D).transpose(1, 2).contiguous()
        return got

    heads = case["heads"]
    pairs = sum(n * m for n, m in zip(s["new"], s["lens"] if case["op"] == "cached" else s["new"]))
    if pairs * heads * D > 1.0e12:
        return None
    result = torch.zeros(starts[-1], heads, D, dtype=torch.float64, device=DEV)
    flat = None
    if case["op"] == "cached":
        flat = {}
        for n in ("k", "v"):
            x = s[n + "_cache"].double()
            if s[n + "_scale"] is not None:
                x = x * s[n + "_scale"].double().unsqueeze(3)
            flat[n] = x
    for b, (n, m) in enumerate(zip(s["new"], s["lens"])):
        lo = starts[b]
        q = s["q"][lo:lo + n].double().reshape(n, heads, D)
        if flat is None:
            k, v = (s[x][lo:lo + n].double().reshape(n, H, D).transpose(0, 1) for x in ("k", "v"))
            ok = torch.ones(n, n, dtype=torch.bool, device=DEV)
            if case["causal"]:
                ok = ok.tril()
            if s["keep"] is not None:
                here = s["keep"][lo:lo + n].bool()
                ok = ok & here[None, :] & here[:, None]
        else:
            def tokens(x, pages, count):
                return x[pages.long()].transpose(0, 1).reshape(H, -1, D)[:, :count]
            mine = s["table"][b, :_pages(m, case["page"])]
            k, v = (tokens(flat[x], mine, m) for x in ("k", "v"))
            if case["prefix"]:
                k, v = (torch.cat((tokens(flat[x], s["prefix"], case["prefix"]), y), 1) for x, y in (("k", k), ("v", v)))
            total = k.shape[1]
            ok = torch.ones(n, total, dtype=torch.bool, device=DEV).tril(total - n)
        for h in range(heads):
            kh, vh = k[h * H // heads], v[h * H // heads]
            z = q[:, h] @ kh.t().contiguous() / math.sqrt(D)
            z = torch.where(ok, z, torch.tensor(-math.inf, dtype=torch.float64, device=DEV))
            e = torch.where(ok, torch.exp(z - z.max(1, keepdim=True).values), torch.zeros((), dtype=torch.float64, device=DEV))
            total_weight = e.sum(1, keepdim=True)
            result[lo:lo + n, h] = (e @ vh.contiguous()) / torch.where(total_weight > 0, total_weight, 1.0)
    return result.reshape(starts[-1], heads * D)
