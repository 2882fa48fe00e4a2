"""The experts' hidden values are float32 between the two products, whatever the weights' type: single hidden values of chosen bits,
every other one zero, on each way through the last product.

A token goes to one expert with weight 1.  Its gate projection is 2^6 (or 2^127), where silu(g) = g / (1 + exp(-g)) is g itself in
float32; its up projection is a sum of products that float32 holds.  All results are exact: there is no tolerance."""
import math

import pytest
import torch

import paper_2308_15949_amd as L

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": E4M3}
# tokens, experts: one token; entries no more than the experts; more entries than experts, more than sixteen of one expert
SIZES = [(1, 4), (4, 4), (7, 3), (40, 5)]


def blocks(n):
    return -(-n // 128)


class Layer:
    """Experts of zeros; x = (1, 2^-10, 2^-14, 1, 0, ...) for every token, the router sends all of them to expert `chosen`."""

    def __init__(self, T, E, C, F, w):
        self.T, self.E, self.C, self.F, self.w, self.chosen = T, E, C, F, w, E - 1
        dt = torch.float32 if w == "f32" else torch.bfloat16
        self.x = torch.zeros(T, C, dtype=dt)
        self.x[:, 0], self.x[:, 1], self.x[:, 2], self.x[:, 3] = 1.0, 2.0 ** -10, 2.0 ** -14, 1.0
        self.router = torch.zeros(E, C, dtype=dt)
        self.router[self.chosen, 0] = 64.0
        self.up, self.down = torch.zeros(E, 2, F, C), torch.zeros(E, C, F)
        self.s_up = self.s_down = None
        if w == "e4m3":
            self.s_up, self.s_down = torch.ones(E, 2, blocks(F), blocks(C)), torch.ones(E, blocks(C), blocks(F))

    def run(self):
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        held = [dev(t) for t in (self.router, self.up.to(TYPES[self.w]), self.down.to(TYPES[self.w]), self.s_up, self.s_down)]
        p = L.make_moe(*held, top_k=1, renormalise=True)
        out = torch.full((self.T, self.C), 7.0).to(self.x.dtype).cuda()
        wt = torch.empty(self.T, 1, device="cuda")
        ids = torch.empty(self.T, 1, device="cuda", dtype=torch.int32)
        L.laud_moe(p, self.x.cuda(), None, out, ids, wt, torch.full((L.moe_workspace(p, self.T),), 255, dtype=torch.uint8, device="cuda"))
        assert bool((ids == self.chosen).all()) and bool((wt == 1).all())
        return out.cpu().float()


@pytest.mark.parametrize("w", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("T,E", SIZES)
@pytest.mark.parametrize("C,F,at,other", [(16, 16, 3, 9), (144, 272, 3, 200), (144, 272, 259, 131), (272, 1040, 1039, 0), (16, 2064, 1500, 1499)])
def test_all_bits_of_a_hidden_value_count(T, E, C, F, at, other, w):
    """Two hidden values that differ in their last bits, with opposite signs in the last product: the difference is the result."""
    m = Layer(T, E, C, F, w)
    e = m.chosen
    m.up[e, 0, (at, other), 0] = 64.0
    m.up[e, 1, (at, other), 0] = 1.0
    m.up[e, 1, (at, other), 3] = 2.0 ** -9
    m.up[e, 1, at, 1], m.up[e, 1, at, 2] = 2.0 ** -9, 2.0 ** -9    # 1 + 2^-9 + 2^-19 + 2^-23: 24 bits, and no sum of two bf16
    sign = 1.0 - 2.0 * (torch.arange(C) % 2)
    m.down[e, :, at], m.down[e, :, other] = sign, -sign
    assert torch.equal(m.run(), (sign * 64 * (2.0 ** -19 + 2.0 ** -23)).expand(T, C))


@pytest.mark.parametrize("w", ["bf16", "f32", "e4m3"])
@pytest.mark.parametrize("T,E", SIZES)
def test_finite_hidden_values_stay_finite(T, E, w):
    """2^128 (1 - 2^-20), which rounds to infinity in bf16."""
    m = Layer(T, E, 16, 272, w)
    e, at = m.chosen, 140
    if w == "e4m3":
        m.up[e, 0, at, 0], m.s_up[e, 0] = 256.0, 2.0 ** 119
        m.s_down[e] = 2.0 ** -64
    else:
        m.up[e, 0, at, 0] = 2.0 ** 127
    m.up[e, 1, at, 0], m.up[e, 1, at, 1] = 2.0, -(2.0 ** -9)
    m.down[e, :, at] = 1.0 if w == "e4m3" else 2.0 ** -64
    ref = torch.full((T, 16), 2.0 ** 64 * (1 - 2.0 ** -20)).to(m.x.dtype).float()
    assert torch.equal(m.run(), ref)


@pytest.mark.parametrize("w", ["bf16", "f32"])
@pytest.mark.parametrize("T,E", SIZES)
@pytest.mark.parametrize("F", [16, 400])
def test_infinite_weights_of_the_last_product(T, E, F, w):
    """Every hidden value is 64, exact in bf16: an infinite weight makes an infinity of its sign, not a NaN."""
    m = Layer(T, E, 24, F, w)
    e = m.chosen
    m.up[e, 0, :, 0], m.up[e, 1, :, 0] = 64.0, 1.0
    m.down[e] = 0.5
    m.down[e, 3, F - 2], m.down[e, 4, 1] = math.inf, -math.inf
    ref = torch.full((T, 24), 32.0 * F)
    ref[:, 3], ref[:, 4] = math.inf, -math.inf
    assert torch.equal(m.run(), ref)
