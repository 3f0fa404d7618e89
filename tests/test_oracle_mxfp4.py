"""Pins of the MXFP4 rule in oracle/paged.py."""

from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle.paged import E2M1, block_codes, mx_values, pack_e2m1, round_e2m1


def test_round_e2m1_is_the_nearest_number():
    """Against a search over all E2M1 numbers; ties go to the code with the even last bit."""
    y = np.concatenate([np.arange(-7 + 2.0 ** -6, 7, 2.0 ** -6), np.random.default_rng(1).uniform(-7, 7, 2000)])
    for v, got in zip(y, round_e2m1(y)):
        near = [(abs(Fraction(float(abs(v))) - Fraction(float(c))), i % 2, c) for i, c in enumerate(E2M1)]
        assert abs(got) == min(near)[2] and got * v >= 0


def test_block_by_hand():
    x = np.zeros(64)
    x[:8] = [6.0, -6.9, 0.25, 0.75, 5.0, 3.5, -2.5, 1.2]          # below 7: 2^0
    x[32:36] = [7.0, 1.0, -0.5, 3.4]                               # 7 itself: 2^1
    codes, byte = block_codes(x)
    np.testing.assert_array_equal(byte, [127, 128])
    np.testing.assert_array_equal(codes[:8], [6, -6, 0, 1, 4, 4, -2, 1])
    np.testing.assert_array_equal(codes[32:36], [4, 0.5, -0.0, 1.5])   # 3.5, .5, -.25 and 1.7
    packed = pack_e2m1(codes)
    np.testing.assert_array_equal(packed[:4], [0x7 | 0xF << 4, 0 | 2 << 4, 6 | 6 << 4, 0xC | 2 << 4])
    np.testing.assert_array_equal(packed[16:18], [6 | 1 << 4, 8 | 3 << 4])
    np.testing.assert_array_equal(mx_values(packed, byte), codes * np.repeat([1.0, 2.0], 32))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_exponents_are_the_least(dtype):
    f = torch.finfo(dtype)
    top = torch.cat([torch.tensor([f.max, f.smallest_normal, f.smallest_normal * f.eps, 7.0, 6.99, 3.5, 3.49, 1.0]),
                     torch.logspace(-4, 4, 50)]).to(dtype).double().numpy()
    x = np.zeros((len(top), 32))
    x[:, 5] = -top
    codes, byte = block_codes(x)
    for a, c, b in zip(top, codes, byte):
        e = int(b) - 127
        assert a < 7 * 2.0 ** e and (e == -127 or a >= 7 * 2.0 ** (e - 1))
        # a 2^-e lies in [3.5, 7), where the numbers are 3, 4 and 6: the furthest from one, relative to itself, is 5.
        assert abs(c[5]) * 2.0 ** e == pytest.approx(a, rel=1 / 5 if e > -127 else 1.0)


def test_special_blocks():
    x = np.zeros((4, 32))
    x[1, 3], x[2, 0], x[3] = np.inf, np.nan, -0.0
    codes, byte = block_codes(x)
    np.testing.assert_array_equal(byte[:, 0], [0, 255, 255, 0])
    assert not codes.any() and np.signbit(codes[3]).all()
    assert np.isnan(mx_values(pack_e2m1(codes), byte)[1:3]).all()


def test_values_of_every_byte():
    codes = np.arange(256, dtype=np.uint8).reshape(16, 16)
    v = mx_values(codes, np.full((16, 1), 127, np.uint8))
    want = np.concatenate([E2M1, -E2M1])
    np.testing.assert_array_equal(v[:, 0::2].ravel(), want[np.arange(256) % 16])
    np.testing.assert_array_equal(v[:, 1::2].ravel(), want[np.arange(256) // 16])
