"""The reference of the cache in blocks by its own definition, on the CPU: rounding against torch's cast, exponents, older tokens."""
import math

import numpy as np
import torch

from oracle import blocks_oracle as BO


def test_codes_are_torchs_nearest():
    g = torch.Generator().manual_seed(1)
    x = torch.cat([torch.randn(4000, generator=g) * s for s in (1e-3, 0.02, 1.0, 100.0)] + [torch.arange(-460, 460).float(), torch.arange(-40, 40).float() / 1024])
    x = x.clamp(-448, 448)
    assert np.array_equal(BO.e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    keep = ~np.isnan(codes)
    assert np.array_equal(BO.e4m3(codes[keep]), codes[keep]) and np.isnan(BO.e4m3(codes[~keep])).all()
    assert BO.e4m3(np.array([1e9, -1e9, math.inf])).tolist() == [448.0, -448.0, 448.0]


def test_exponents_are_the_least():
    assert BO.least_exponent(np.zeros(3)) == BO.LEAST and BO.least_exponent(np.array([math.nan, math.inf])) == BO.LEAST
    for top, e in ((448.0, 0), (448.5, 1), (224.0, -1), (1.0, -8), (1.75, -8), (1.76, -7), (3.3895313892515355e38, 120)):
        assert BO.least_exponent(np.array([0.25, -top])) == e


def test_older_tokens_follow_a_larger_exponent():
    c = BO.Blocks(2, 1, 16, 2)
    c.put([1], 0, np.array([[[0.5, 448.0 * 2 ** -20]]]))
    c.put([1], 1, np.array([[[64.0, 0.0]]]))                     # 2^7 times as large
    assert c.e[1, 0, 0] == -2
    assert c.values([1], 2)[:, 0].tolist() == [[0.5, 2.0 ** -11], [64.0, 0.0]]       # 448 2^-20 = 1.75 2^-12: the nearest of subnormal codes, 2^-9 2^-2
    c.put([1], 16, np.ones((1, 1, 2)))                           # no page: nothing
    assert c.e[0, 0, 0] == BO.LEAST
