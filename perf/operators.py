"""Workloads of the token operators: norms around a block with gate and residual scale, 8-bit quantisation in blocks of 128, the
matrix product of 8-bit operands with a scale for each block of 128, and the mixture-of-experts layer for a few tokens.

A case is a dict of plain values.  listed() names the standing ones, draw() gives more of the same ranges, prepare() makes what a
program has in hand before the call, run() is one pass through an operator: in its plain form, elementary operations in 32 bits
(own = False), or through this package's entry points (own = True).  work() is what a pass cannot do without, exact() the result
in 64 bits from the definition.

Definitions
  norm    p = N(y; post) or y;  r = keep ? alpha x + beta gate p : x;  out = r;  z = N(r; pre), in x's type or in 8 bits
          N is v / rms(v) * w + b or (v - mean) / std(v) * w + b
  quant   blocks of 1 x 128 (activations) or 128 x 128 (weights): s = max(max|x| / 448, 2^-126), q = e4m3(x / s)
  matmul  out[m, n] = sum_k a[m, k] sa[m, k / 128] b[n, k] sb[n / 128, k / 128]
  moe     softmax of x Wr^T, the top_k experts of a token, sum of weight * (silu(x Wg^T) * (x Wu^T)) Wd^T over them;
          a token whose keep is 0 gets zeros and experts -1
8-bit results are returned as float8 tensors (the values of the codes) beside their scales.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
BLK = 128
EPS = 1e-5


# ----- cases ------------------------------------------------------------------------------------------------------------
def listed() -> list[dict]:
    return [
        # the step of a decoder on four sequences: one launch whose latency is everything
        dict(name="norm_rows4", op="norm", rows=4, C=2048, dtype="bf16", kind="rms", post=True, pre=True, z="same", keep=1.0,
             groups=0),
        # an odd number of image tokens (14 x 14 and one more) of five samples in float32, layer norms with biases, a gate per sample
        # and channel, a third of the tokens skipped
        dict(name="norm_f32_tokens", op="norm", rows=985, C=1064, dtype="f32", kind="layer", post=True, pre=True, z="same", keep=0.66,
             groups=5),
        # a server batch: residual stream in and out, next block's input straight in 8 bits
        dict(name="norm_batch_e4m3", op="norm", rows=16384, C=4096, dtype="bf16", kind="rms", post=True, pre=True, z="e4m3",
             keep=0.75, groups=0),
        # activations of a small float32 model, a width that ends inside a block
        dict(name="quant_f32_ragged", op="quant", rows=197, cols=1480, dtype="f32", block_rows=1),
        # activations of a server batch
        dict(name="quant_batch", op="quant", rows=16384, cols=4096, dtype="bf16", block_rows=1),
        # one token through a projection: the weights are read for one row
        dict(name="matmul_row1", op="matmul", M=1, N=4096, K=4096, out="bf16"),
        # image tokens of one sample, float32 results
        dict(name="matmul_tokens197", op="matmul", M=197, N=2048, K=1024, out="f32"),
        # sizes that end inside every tile and block
        dict(name="matmul_odd", op="matmul", M=1003, N=2120, K=2000, out="bf16"),
        # a server batch through a feed-forward projection
        dict(name="matmul_batch", op="matmul", M=8192, N=8192, K=4096, out="bf16"),
        # one token: eight experts' weights are read, for one row each
        dict(name="moe_token1", op="moe", T=1, E=64, top_k=8, C=2048, F=1024, dtype="bf16", w="bf16", keep=1.0, renorm=True),
        # a few tokens, experts in 8 bits, widths that end inside a block, one token in eight skipped
        dict(name="moe_tokens16_e4m3", op="moe", T=16, E=64, top_k=6, C=2048, F=1424, dtype="bf16", w="e4m3", keep=0.875,
             renorm=False),
        # the upper end of a few: nearly every expert is met
        dict(name="moe_tokens64", op="moe", T=64, E=64, top_k=8, C=2048, F=1024, dtype="bf16", w="bf16", keep=1.0, renorm=True),
    ]


def _log_int(rng, lo: int, hi: int, step: int = 1) -> int:
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))) / step)) * step
    v -= step if v == 3072 else 0  # (a width that no configuration here has)
    return max(lo, min(hi, v))


def draw(rng) -> dict:
    op = rng.choice(("norm", "norm", "quant", "matmul", "matmul", "moe", "moe"))
    if op == "norm":
        C = _log_int(rng, 64, 8192, 8)
        rows = _log_int(rng, 1, min(16384, 16384 * 4096 // C))
        groups = rng.choice((0, 1, rng.randint(1, min(rows, 16))))
        return dict(op=op, rows=rows, C=C, dtype=rng.choice(("bf16", "bf16", "f32")), kind=rng.choice(("rms", "layer")),
                    post=rng.random() < 0.7, pre=rng.random() < 0.8, z=rng.choice(("same", "same", "e4m3")),
                    keep=rng.choice((1.0, 1.0, round(rng.uniform(0.0, 0.9), 2))), groups=groups)
    if op == "quant":
        cols = _log_int(rng, 64, 8192, 8)
        rows = _log_int(rng, 1, min(16384, 16384 * 4096 // cols))
        return dict(op=op, rows=rows, cols=cols, dtype=rng.choice(("bf16", "bf16", "f32")), block_rows=rng.choice((1, 1, BLK)))
    if op == "matmul":
        while True:
            M, N, K = _log_int(rng, 1, 8192), _log_int(rng, 64, 8192, 8), _log_int(rng, 64, 8192, 16)
            if M * N * K <= 8192 * 8192 * 4096:
                return dict(op=op, M=M, N=N, K=K, out=rng.choice(("bf16", "bf16", "f32")))
    while True:
        E, C, F = rng.choice((4, 8, 16, 30, 64, 128)), _log_int(rng, 256, 4096, 16), _log_int(rng, 128, 2048, 16)
        if E * C * F <= 64 * 2048 * 1024:
            break
    w = rng.choice(("bf16", "e4m3", "e4m3", "f32"))
    return dict(op=op, T=_log_int(rng, 1, 64), E=E, top_k=rng.randint(1, min(E, 8)), C=C, F=F, dtype="f32" if w == "f32" else "bf16",
                w=w, keep=rng.choice((1.0, 1.0, round(rng.uniform(0.3, 0.9), 2))), renorm=rng.random() < 0.5)


# ----- inputs -----------------------------------------------------------------------------------------------------------
def _blocks(n: int) -> int:
    return -(-n // BLK)


class _Rand:
    def __init__(self, seed: int):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device=DEV)

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device=DEV)

    def features(self, rows: int, cols: int, dtype):
        """Activations of a trained model: channels of different size, a few of them large."""
        size = torch.exp(0.5 * self.normal(cols)) * torch.where(self.uniform(cols) < 0.01, 8.0, 1.0)
        return (self.normal(rows, cols) * size).to(dtype)

    def keep(self, n: int, share: float):
        return None if share >= 1.0 else (self.uniform(n) < share).to(torch.uint8)

    def codes(self, *shape):
        """8-bit weights as quantisation leaves them: normal values, the largest of a block near the type's largest."""
        return (self.normal(*shape) * 128.0).clamp_(-448.0, 448.0).to(E4M3)

    def scales(self, k: int, *shape):
        """... and their scales: weights of about 1 / sqrt(k)."""
        return torch.exp(0.2 * self.normal(*shape)) / (128.0 * math.sqrt(k))


def prepare(case: dict, seed: int) -> dict:
    r = _Rand(seed)
    s = {"case": case}
    if case["op"] == "norm":
        R, C, dt = case["rows"], case["C"], TYPES[case["dtype"]]
        s["x"], s["y"] = r.features(R, C, dt), r.features(R, C, dt)
        layer = case["kind"] == "layer"
        for k in ("post", "pre"):
            s[k + "_w"] = 1 + 0.1 * r.normal(C) if case[k] else None
            s[k + "_b"] = 0.1 * r.normal(C) if case[k] and layer else None
        s["keep"] = r.keep(R, case["keep"])
        s["gate"] = 0.5 * r.normal(case["groups"], C) if case["groups"] else None
        s["alpha"], s["beta"] = 1.0, 0.5
        s["out"] = torch.empty_like(s["x"])
        if case["pre"]:
            s["z"] = torch.empty(R, C, device=DEV, dtype=E4M3 if case["z"] == "e4m3" else dt)
            s["zs"] = torch.empty(R, _blocks(C), device=DEV) if case["z"] == "e4m3" else None
    elif case["op"] == "quant":
        R, C = case["rows"], case["cols"]
        s["x"] = r.features(R, C, TYPES[case["dtype"]])
        s["q"] = torch.empty(R, C, device=DEV, dtype=E4M3)
        s["s"] = torch.empty(-(-R // case["block_rows"]), _blocks(C), device=DEV)
    elif case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"], s["sa"] = r.codes(M, K), torch.exp(0.5 * r.normal(M, _blocks(K))) / 128.0
        s["b"], s["sb"] = r.codes(N, K), r.scales(K, _blocks(N), _blocks(K))
        s["out"] = torch.empty(M, N, device=DEV, dtype=TYPES[case["out"]])
    else:
        T, E, C, F, dt = case["T"], case["E"], case["C"], case["F"], TYPES[case["dtype"]]
        s["x"] = r.normal(T, C).to(dt)
        s["router"] = (2.0 * r.normal(E, C) / math.sqrt(C)).to(dt)
        if case["w"] == "e4m3":
            s["up"], s["s_up"] = r.codes(E, 2, F, C), r.scales(C, E, 2, _blocks(F), _blocks(C))
            s["down"], s["s_down"] = r.codes(E, C, F), r.scales(F, E, _blocks(C), _blocks(F))
        else:
            s["up"], s["s_up"] = (r.normal(E, 2, F, C) / math.sqrt(C)).to(dt), None
            s["down"], s["s_down"] = (r.normal(E, C, F) / math.sqrt(F)).to(dt), None
        s["keep"] = r.keep(T, case["keep"])
        s["out"] = torch.empty(T, C, device=DEV, dtype=dt)
        s["experts"] = torch.empty(T, case["top_k"], device=DEV, dtype=torch.int32)
        s["weights"] = torch.empty(T, case["top_k"], device=DEV)
    return s


# ----- one pass ---------------------------------------------------------------------------------------------------------
def run(state: dict):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state)


def _norm32(v, kind: str, w, b):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * w
    return v if b is None else v + b


def _quant32(v, block_rows: int = 1):
    """The codes' values in 8 bits and their scales."""
    R, C = v.shape
    rb, cb = -(-R // block_rows), _blocks(C)
    v = torch.nn.functional.pad(v, (0, cb * BLK - C, 0, rb * block_rows - R)).view(rb, block_rows, cb, BLK)
    largest = torch.tensor(448.0, device=v.device)
    s = (v.abs().amax((1, 3)) / largest).clamp_min(2.0 ** -126)
    return (v / s[:, None, :, None]).view(rb * block_rows, cb * BLK)[:R, :C].to(E4M3), s


def _plain_norm(s):
    c = s["case"]
    x, p = s["x"].float(), s["y"].float()
    if c["post"]:
        p = _norm32(p, c["kind"], s["post_w"], s["post_b"])
    if s["gate"] is not None:
        each = -(-c["rows"] // c["groups"])
        p = p * s["gate"].repeat_interleave(each, 0)[: c["rows"]]
    r = s["alpha"] * x + s["beta"] * p
    if s["keep"] is not None:
        r = torch.where(s["keep"][:, None] != 0, r, x)
    got = {"out": r.to(s["x"].dtype)}
    if c["pre"]:
        z = _norm32(r, c["kind"], s["pre_w"], s["pre_b"])
        if c["z"] == "e4m3":
            got["z"], got["z_scale"] = _quant32(z)
        else:
            got["z"] = z.to(s["x"].dtype)
    return got


def _plain_quant(s):
    q, scale = _quant32(s["x"].float(), s["case"]["block_rows"])
    return {"q": q, "scale": scale}


def _wide(scale, rows: int, cols: int, block_rows: int):
    if block_rows > 1:
        scale = scale.repeat_interleave(block_rows, -2)[..., :rows, :]
    return scale.repeat_interleave(BLK, -1)[..., :cols]


def _plain_matmul(s):
    c = s["case"]
    a = s["a"].float() * _wide(s["sa"], c["M"], c["K"], 1)
    b = s["b"].float() * _wide(s["sb"], c["N"], c["K"], BLK)
    return (a @ b.t()).to(s["out"].dtype)


def _plain_moe(s):
    c = s["case"]
    T, E, k, C, F = c["T"], c["E"], c["top_k"], c["C"], c["F"]
    x = s["x"].float()
    logits = x @ s["router"].float().t()
    order = torch.sort(logits, dim=-1, descending=True, stable=True).indices[:, :k]
    experts = torch.sort(order, -1).values
    weights = torch.softmax(logits, -1).gather(1, experts)
    if c["renorm"]:
        weights = weights / weights.sum(-1, keepdim=True)
    if s["keep"] is not None:
        weights = torch.where(s["keep"][:, None] != 0, weights, 0.0)

    def expert_weights(ids):
        """The chosen experts' matrices in 32 bits (ids None: all of them, in order)."""
        take = (lambda t: t) if ids is None else (lambda t: t.view(torch.uint8)[ids].view(E4M3) if t.dtype == E4M3 else t[ids])
        up, down = take(s["up"]).float(), take(s["down"]).float()
        if s["s_up"] is not None:
            up = up * _wide(take(s["s_up"]), F, C, BLK)
            down = down * _wide(take(s["s_down"]), C, F, BLK)
        return up, down

    if T * k < E:  # fewer choices than experts: each choice with its expert's matrices
        up, down = expert_weights(experts.reshape(-1))
        xs = x.repeat_interleave(k, 0)[:, :, None]
        h = torch.nn.functional.silu(torch.bmm(up[:, 0], xs)) * torch.bmm(up[:, 1], xs)
        y = torch.bmm(down, h).view(T, k, C)
        out = (weights[:, :, None] * y).sum(1)
    else:          # every expert on every token, weighted with zero where it was not chosen
        up, down = expert_weights(None)
        h = torch.matmul(up.view(E * 2 * F, C), x.t()).view(E, 2, F, T)
        h = torch.nn.functional.silu(h[:, 0]) * h[:, 1]
        share = torch.zeros(T, E, device=x.device).scatter_(1, experts, weights)
        h = h * share.t()[:, None, :]
        out = torch.bmm(down, h).sum(0).t()
    if s["keep"] is not None:
        experts = torch.where(s["keep"][:, None] != 0, experts, -1)
    return {"out": out.to(s["x"].dtype), "experts": experts.to(torch.int32), "weights": weights}


_PLAIN = {"norm": _plain_norm, "quant": _plain_quant, "matmul": _plain_matmul, "moe": _plain_moe}


def _own_norm(s):
    from paper_2308_15949_amd import binding as B
    c = s["case"]
    if "p" not in s:
        s["p"] = B.make_norm_block(c["C"], s["x"].dtype, c["kind"], EPS, s["post_w"], s["post_b"], s["pre_w"], s["pre_b"], s["alpha"],
                                   s["beta"])
    each = -(-c["rows"] // c["groups"]) if c["groups"] else 0
    B.laud_norm_residual(s["p"], s["x"], s["y"], s["keep"], s["gate"], each, s["out"], s.get("z"), s.get("zs"))
    got = {"out": s["out"]}
    if c["pre"]:
        got["z"] = s["z"]
        if c["z"] == "e4m3":
            got["z_scale"] = s["zs"]
    return got


def _own_quant(s):
    from paper_2308_15949_amd import binding as B
    B.laud_quantize_e4m3(s["x"], s["q"], s["s"], s["case"]["block_rows"])
    return {"q": s["q"], "scale": s["s"]}


def _own_matmul(s):
    from paper_2308_15949_amd import binding as B
    c = s["case"]
    if "ws" not in s:
        n = B.matmul_e4m3_workspace(c["M"], c["N"], c["K"])
        s["ws"] = torch.empty(n, dtype=torch.uint8, device=DEV) if n else None
    B.laud_matmul_e4m3(s["a"], s["sa"], s["b"], s["sb"], s["out"], s["ws"])
    return s["out"]


def _own_moe(s):
    from paper_2308_15949_amd import binding as B
    c = s["case"]
    if "p" not in s:
        s["p"] = B.make_moe(s["router"], s["up"], s["down"], s["s_up"], s["s_down"], c["top_k"], c["renorm"], 1.0)
        s["ws"] = torch.empty(B.moe_workspace(s["p"], c["T"]), dtype=torch.uint8, device=DEV)
    B.laud_moe(s["p"], s["x"], s["keep"], s["out"], s["experts"], s["weights"], s["ws"])
    return {"out": s["out"], "experts": s["experts"], "weights": s["weights"]}


_OWN = {"norm": _own_norm, "quant": _own_quant, "matmul": _own_matmul, "moe": _own_moe}


# ----- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case: dict) -> dict:
    if case["op"] == "norm":
        R, C, e = case["rows"], case["C"], 4 if case["dtype"] == "f32" else 2
        kept = R * case["keep"]  # (a skipped row's block output is not needed)
        vectors = (2 if case["kind"] == "layer" else 1) * (case["post"] + case["pre"]) + case["groups"]
        nbytes = R * C * 2 * e + kept * C * e + 4 * C * vectors + (R if case["keep"] < 1 else 0)
        if case["pre"]:
            nbytes += R * C + 4 * R * _blocks(C) if case["z"] == "e4m3" else R * C * e
        return {"bytes": nbytes, "flops": R * C * (4 + 6 * (case["post"] + case["pre"]))}
    if case["op"] == "quant":
        R, C, e = case["rows"], case["cols"], 4 if case["dtype"] == "f32" else 2
        return {"bytes": R * C * (e + 1) + 4 * _blocks(C) * -(-R // case["block_rows"]), "flops": 3 * R * C}
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": M * K + N * K + 4 * (M + _blocks(N)) * _blocks(K) + M * N * (4 if case["out"] == "f32" else 2),
                "flops": 2 * M * N * K}
    T, E, k, C, F = case["T"], case["E"], case["top_k"], case["C"], case["F"]
    kept, e = T * case["keep"], 4 if case["dtype"] == "f32" else 2
    met = E * (1 - (1 - k / E) ** kept)  # experts that some token chose, on average
    each = 3 * C * F * (1 if case["w"] == "e4m3" else e)
    if case["w"] == "e4m3":
        each += 4 * (2 * _blocks(F) * _blocks(C) + _blocks(C) * _blocks(F))
    return {"bytes": met * each + E * C * e + 2 * T * C * e + 8 * T * k, "flops": 6 * kept * k * C * F + 2 * kept * E * C}


# ----- the result in 64 bits, from the definitions --------------------------------------------------------------------------
def _exact_norm_of(v, kind, w, b):
    centre = v.sum(1, keepdim=True) / v.shape[1] if kind == "layer" else 0.0
    spread = ((v - centre) ** 2).sum(1, keepdim=True) / v.shape[1]
    u = (v - centre) / (spread + EPS).sqrt() * w.double()
    return u if b is None else u + b.double()


def _exact_codes(v, block_rows):
    """Rows of blocks one after the other; scales are float32 by definition, quotients in 64 bits."""
    R, C = v.shape
    codes, scales = torch.empty_like(v), torch.empty(-(-R // block_rows), _blocks(C), dtype=torch.float64, device=v.device)
    for j in range(_blocks(C)):
        part = v[:, j * BLK:(j + 1) * BLK]
        top = part.abs().max(1).values
        if block_rows > 1:
            top = torch.stack([t.max() for t in top.split(block_rows)])
        scale = (top / 448.0).float().double().clamp(min=2.0 ** -126)
        scales[:, j] = scale
        codes[:, j * BLK:(j + 1) * BLK] = (part / scale.repeat_interleave(block_rows)[:R, None]).to(E4M3).double()
    return codes, scales


def exact(case: dict, seed: int):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x, branch, rows = s["x"].double(), s["y"].double(), case["rows"]
        if case["post"]:
            branch = _exact_norm_of(branch, case["kind"], s["post_w"], s["post_b"])
        if case["groups"]:
            of = torch.arange(rows, device=DEV) // (-(-rows // case["groups"]))
            branch = branch * s["gate"].double()[of]
        r = s["alpha"] * x + s["beta"] * branch
        if s["keep"] is not None:
            skipped = s["keep"] == 0
            r[skipped] = x[skipped]
        got = {"out": r}
        if case["pre"]:
            z = _exact_norm_of(r, case["kind"], s["pre_w"], s["pre_b"])
            if case["z"] == "e4m3":
                got["z"], got["z_scale"] = _exact_codes(z, 1)
            else:
                got["z"] = z
        return got
    if case["op"] == "quant":
        codes, scales = _exact_codes(s["x"].double(), case["block_rows"])
        return {"q": codes, "scale": scales}
    if case["op"] == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        out = torch.zeros(M, N, dtype=torch.float64, device=DEV)
        for j in range(_blocks(K)):
            part = s["a"][:, j * BLK:(j + 1) * BLK].double() @ s["b"][:, j * BLK:(j + 1) * BLK].double().t().contiguous()
            part *= s["sa"][:, j, None].double()
            part *= s["sb"][:, j].double().repeat_interleave(BLK)[None, :N]
            out += part
        return out
    T, k, C, F = case["T"], case["top_k"], case["C"], case["F"]
    x = s["x"].double()
    logits = x @ s["router"].double().t().contiguous()
    share = torch.exp(logits - logits.max(1, keepdim=True).values)
    share = share / share.sum(1, keepdim=True)
    chosen = torch.sort(torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k], 1).values
    weights = share.gather(1, chosen)
    if case["renorm"]:
        weights = weights / weights.sum(1, keepdim=True)
    if s["keep"] is not None:
        weights = weights * (s["keep"] != 0).double()[:, None]

    def matrix(w, scale):
        w = w.double()
        if scale is not None:
            i, j = (torch.arange(n, device=DEV) // BLK for n in w.shape)
            w = w * scale.double()[i][:, j]
        return w

    out = torch.zeros(T, C, dtype=torch.float64, device=DEV)
    for e in chosen.unique().tolist():
        at, slot = (chosen == e).nonzero(as_tuple=True)
        gate, up, down = (matrix(s[n][e] if i is None else s[n][e, i],
                                 None if s["s_" + n] is None else (s["s_" + n][e] if i is None else s["s_" + n][e, i]))
                          for n, i in (("up", 0), ("up", 1), ("down", None)))
        g = x[at] @ gate.t().contiguous()
        h = g / (1 + torch.exp(-g)) * (x[at] @ up.t().contiguous())
        out[at] += weights[at, slot][:, None] * (h @ down.t().contiguous())
    return {"out": out, "experts": None, "weights": weights}
