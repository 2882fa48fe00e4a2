"""Quantisation of blocks of any size: codes are those of the float32 quotient x / scale, also where the scale is so small that what a
quotient leaves over is no float any more.  Elements stand on and beside the middle between two codes, where one bit decides."""
import numpy as np
import pytest
import torch

import paper_2308_15949_amd as L

pytestmark = pytest.mark.gpu
E4M3 = torch.float8_e4m3fn


def blocks_of(exponents, seed, each=64):
    """Rows of one block of 128 float32, whose scales have the given exponents."""
    rng = np.random.default_rng(seed)
    codes = np.arange(127, dtype=np.uint8)
    values = torch.from_numpy(codes).view(E4M3).double().numpy()
    middle = (values[1:] + values[:-1]) / 2
    rows = []
    for e in exponents:
        for _ in range(each):
            s = np.float32(np.ldexp(1 + rng.random(), e))
            f = (rng.choice(middle, 128) * np.float64(s)).astype(np.float32)
            f = (f.view(np.int32) + rng.integers(-2, 3, 128).astype(np.int32) * (f.view(np.int32) > 4)).view(np.float32)
            f[rng.integers(128)] = np.float32(448 * np.float64(s))
            rows.append(f * rng.choice(np.array([-1, 1], np.float32), 128))
    return np.stack(rows)


@pytest.mark.parametrize("exponents", [range(-130, -110), range(-110, -90), range(-90, -50), range(-50, 20), range(20, 118)])
def test_codes_are_those_of_the_quotient(exponents):
    x = blocks_of(exponents, abs(exponents[0]))
    q, s = torch.empty(*x.shape, device="cuda", dtype=E4M3), torch.empty(len(x), 1, device="cuda")
    L.laud_quantize_e4m3(torch.from_numpy(x).cuda(), q, s, 1)
    scale = np.maximum(np.abs(x).max(1, keepdims=True) / np.float32(448), np.float32(2.0 ** -126))
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.isfinite(scale).all()
    ref = torch.from_numpy(x / scale).to(E4M3)
    assert torch.equal(q.cpu().view(torch.uint8), ref.view(torch.uint8))
