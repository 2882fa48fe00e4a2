"""Numbers of a batch that 32 bits do not hold, and as many sequences as a launch takes."""
import pytest
import torch

import paper_2308_15949_amd as L
from test_gpu_attention import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [(1 << 32) + 16, 1 << 31, -1])
def test_prefixes_of_more_than_32_bits_are_refused(tokens):
    batch = ints([0, 1]), ints([5]), ints([[0]]), ints([1])
    assert L.make_batch(*batch, 16).prefix_len == 16
    with pytest.raises(L.LaudError):
        L.make_batch(*batch, tokens)


def test_a_million_sequences_of_one_token():
    """More workgroups of sixteen rows than one launch takes, but not of 128.  A token alone has the weight 1: its value is the result."""
    n, heads, D = 1000000, 16, 8
    q, k, v = (torch.randn(n, heads * D, generator=torch.Generator("cuda").manual_seed(i), device="cuda").to(torch.bfloat16) for i in range(3))
    out = torch.zeros_like(q)
    L.laud_attention(L.make_heads(heads, heads, D, torch.bfloat16, True), torch.arange(n + 1, dtype=torch.int32, device="cuda"), q, k, v, None, out)
    assert torch.equal(out, v)
