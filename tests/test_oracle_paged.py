"""Pins of oracle/paged.py, and the arithmetic of the row quantisation that the kernels use."""

import os
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle.paged import TOP, attended, paged_decode, round_e4m3, row_codes, slot_of

HERE = os.path.dirname(os.path.abspath(__file__))


def test_round_e4m3_is_torchs_conversion():
    grid = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    grid = torch.unique(grid[torch.isfinite(grid)])
    mid = (grid[1:] + grid[:-1]) / 2                       # ties
    y = torch.cat([grid, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), torch.linspace(-448, 448, 9001).double()])
    want = y.float().to(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(round_e4m3(y.float().double().numpy()), want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_row_codes_against_fractions(fmt):
    """Codes of the exact rational quotient, on rows with many ties (x = a / 2, a = 127 2^k)."""
    rng = np.random.default_rng(3)
    rows = [np.array([1.0, 0.5, -0.5, 0.25, 0.75, 1 / 3]).astype(np.float16),
            np.array([127.0, 63.5, 62.5, -0.5, 1.5, 100.25]).astype(np.float16)]
    rows += [rng.standard_normal(6).astype(np.float16) for _ in range(50)]
    for x in rows:
        codes, scale = row_codes(x, fmt)
        a = max(Fraction(float(abs(v))) for v in x)
        for v, c in zip(x, codes):
            y = Fraction(float(v)) * int(TOP[fmt]) / a
            if fmt == "int8":
                assert c == round(y)                     # half to even
            else:
                near = [Fraction(float(round_e4m3(np.float64(y)) + k)) for k in (0,)][0]
                step = Fraction(2) ** (max(np.frexp(float(y))[1], -5) - 4)
                assert near == round(y / step) * step == Fraction(float(c))
        assert scale == np.float32(float(a)) / np.float32(TOP[fmt])


def test_row_codes_special_rows():
    for fmt in TOP:
        codes, scale = row_codes(np.zeros((2, 4)), fmt)
        assert not codes.any() and not scale.any()
        codes, scale = row_codes(np.array([[1.0, np.inf], [np.nan, 1.0], [3.0, -3.0]]), fmt)
        assert not codes[:2].any() and np.isnan(scale[:2]).all()
        np.testing.assert_array_equal(codes[2], [TOP[fmt], -TOP[fmt]])


def test_slots_by_hand():
    table = np.array([[4, -1, 2], [9, 0, 1]])
    assert slot_of(table, 5, 16, 0, 0) == (4, 0)
    assert slot_of(table, 5, 16, 0, 16) is None           # no page
    assert slot_of(table, 5, 16, 0, 47) == (2, 15)
    assert slot_of(table, 5, 16, 0, 48) is None and slot_of(table, 5, 16, 0, -1) is None
    assert slot_of(table, 5, 16, 1, 3) is None            # a page past the pool
    ids, slots = attended([34, 99], table, 5, 16, 0, 20)
    np.testing.assert_array_equal(ids, [4, 4, 2, 2])       # tokens 14, 15 and 32, 33
    np.testing.assert_array_equal(slots, [14, 15, 0, 1])


def test_decode_is_torchs_attention():
    rng = np.random.default_rng(0)
    B, Hq, Hk, d, page, per = 2, 6, 2, 8, 16, 3
    K, V = (rng.standard_normal((B * per, Hk, page, d)) for _ in range(2))
    Q = rng.standard_normal((B, Hq, d))
    table = rng.permutation(B * per).reshape(B, per)
    O, lse, mass, reach = paged_decode(Q, K, V, [40, 17], table, 0.3)
    for b, L in enumerate([40, 17]):
        k, v = (torch.from_numpy(x[table[b]].transpose(1, 0, 2, 3).reshape(Hk, -1, d)[:, :L]) for x in (K, V))
        q = torch.from_numpy(Q[b]).view(Hk, Hq // Hk, d)
        want = torch.nn.functional.scaled_dot_product_attention(q, k, v, scale=0.3).reshape(Hq, d).numpy()
        np.testing.assert_allclose(O[b], want, rtol=1e-12)
        s = 0.3 * (q @ k.transpose(1, 2)).reshape(Hq, -1)
        np.testing.assert_allclose(lse[b], torch.logsumexp(s, -1).numpy(), rtol=1e-12)
    assert (np.abs(O) <= mass).all() and (np.abs(reach) > 0).all()
    O, lse, _, _ = paged_decode(Q, K, V, [0, -3], table, 0.3)
    assert not O.any() and np.isneginf(lse).all()


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_row_quotient_is_exact(tmp_path):
    """tests/c/row_quotient_check.c: the kernels' quotient top x / a for every pair of 11-bit numbers."""
    exe = tmp_path / "row_quotient_check"
    subprocess.run(["gcc", "-O2", "-ffp-contract=off", "-o", str(exe),
                    os.path.join(HERE, "c", "row_quotient_check.c"), "-lm"], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    assert "mismatches 0 wrong_codes 0" in out.stdout
    assert int(out.stdout.split()[1]) > 25 * 10 ** 7
