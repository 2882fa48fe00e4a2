"""Numbers of a batch that 32 bits do not hold."""
import pytest

import paper_2308_15949_amd as L
from test_gpu_attention import ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [(1 << 32) + 16, 1 << 31, -1])
def test_prefixes_of_more_than_32_bits_are_refused(tokens):
    batch = ints([0, 1]), ints([5]), ints([[0]]), ints([1])
    assert L.make_batch(*batch, 16).prefix_len == 16
    with pytest.raises(L.LaudError):
        L.make_batch(*batch, tokens)
