"""The 8-bit layer's oracle against torch's e4m3, hand cases and brute force (CPU)."""
import numpy as np
import torch

from oracle import fp8_oracle as orc


def test_values_and_rounding_are_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(orc.decode(codes), want)
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.normal(0, 1, 2000), rng.uniform(-448, 448, 2000), rng.normal(0, 2.0 ** -8, 2000), orc.VALUES, -orc.VALUES,
                        (orc.VALUES[1:] + orc.VALUES[:-1]) / 2]).astype(np.float32)      # the midpoints: ties
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(orc.encode(v), want)


def test_scales_are_the_smallest_that_hold_the_block():
    for top in (448.0, 448.5, 224.0, 1.0, 3.5, 3.5000001, 2.0 ** -20, 1e30):
        s = orc.block_scale([[top, -top / 3, 0.0]])
        assert np.log2(s) == int(np.log2(s)) and top / s <= 448 < 2 * top / s
    assert orc.block_scale([[0.0, 0.0]]) == 1.0
    assert orc.block_scale([[np.inf, 7.0, np.nan]]) == orc.block_scale([[7.0]])
    assert orc.block_scale([[2.0 ** -140]]) == 2.0 ** -126


def test_exactly_representable_layers_come_back():
    rng = np.random.default_rng(2)
    w = orc.VALUES[rng.integers(0, 127, (5, 144))] * rng.choice([-1.0, 1.0], (5, 144)) * 2.0 ** -7
    w[0, 0], w[0, 130] = 448 * 2.0 ** -7, 448 * 2.0 ** -7
    codes, scales = orc.quantize(w)
    assert (scales == 2.0 ** -7).all()
    x = np.eye(144)[:3]
    y, mag = orc.linear(x, codes, scales)
    np.testing.assert_array_equal(y, w[:, :3].T)
    np.testing.assert_array_equal(mag, np.abs(y))
