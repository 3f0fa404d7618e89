"""Pins of oracle/rotary.py, and the library's frequencies (host only)."""

import math
import os

import numpy as np
import pytest

import paper_2608_17336_amd as tm
from oracle.rotary import frequencies, pair_channels, rotary

built = pytest.mark.skipif(not os.path.exists(tm.library_path()), reason="libtilemix.so not built (run __graft_entry__.build())")


def test_by_hand():
    x = np.array([[[1.0, 0.0, 0.0, 2.0, 5.0, 6.0]]])
    f = np.array([math.pi / 2, math.pi])                         # a quarter and half a turn per position
    np.testing.assert_allclose(rotary(x, np.array([1]), f, "half")[0, 0], [0, 0, 1, -2, 5, 6], atol=1e-15)
    np.testing.assert_allclose(rotary(x, np.array([1]), f, "interleaved", g=2.0)[0, 0], [0, 2, 0, -4, 5, 6], atol=1e-15)
    np.testing.assert_allclose(rotary(x, np.array([1]), f, "interleaved", inverse=True)[0, 0], [0, -1, 0, -2, 5, 6], atol=1e-15)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_scores_depend_on_the_distance_alone(layout):
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 1, 1, 64))
    f, _ = frequencies(48, 10000.0)
    s = [np.sum(rotary(q, np.array([p + 13]), f, layout) * rotary(k, np.array([p]), f, layout)) for p in (0, 1, 999)]
    np.testing.assert_allclose(s, s[0], rtol=1e-12)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_inverse_is_the_gradient(layout):
    """d/dx of <w, rotary(x)> is rotary^-1(w), with the same g; by differences, too."""
    rng = np.random.default_rng(2)
    x, w = rng.standard_normal((2, 3, 2, 16))
    pos, (f, _) = np.array([0, 5, 70]), frequencies(12, 100.0)
    grad = rotary(w, pos, f, layout, 1.3, inverse=True)
    np.testing.assert_allclose(np.sum(w * rotary(x, pos, f, layout, 1.3)), np.sum(grad * x), rtol=1e-12)
    for at in [(0, 0, 1), (1, 1, 7), (2, 0, 11), (2, 1, 15)]:
        e = np.zeros_like(x)
        e[at] = 0.5
        diff = np.sum(w * (rotary(x + e, pos, f, layout, 1.3) - rotary(x - e, pos, f, layout, 1.3)))
        assert diff == pytest.approx(grad[at], rel=1e-12)


def test_pairs_cover_the_channels():
    for r in (2, 6, 64):
        for layout in ("half", "interleaved"):
            a, b = pair_channels(r, layout)
            assert sorted([*a, *b]) == list(range(r))


@built
@pytest.mark.parametrize("kw", [dict(), dict(base=500.0), dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0),
                                dict(scaling="yarn", factor=16.0, original_len=4096),
                                dict(scaling="yarn", factor=2.5, original_len=100, beta_fast=8.0, beta_slow=0.5)])
@pytest.mark.parametrize("r", [4, 30, 64, 128])
def test_library_frequencies(kw, r):
    f, g = tm.tilemix_rotary_frequencies(r, device="cpu", **kw)
    want, g_want = frequencies(r, **{"base": 10000.0, **kw})
    np.testing.assert_allclose(f.numpy(), want, rtol=1e-13)     # two pow() and their products in float64
    assert g == pytest.approx(g_want, rel=2.0 ** -24)


def test_yarn_keeps_the_fast_and_divides_the_slow():
    f, _ = frequencies(128, 10000.0)
    y, g = frequencies(128, 10000.0, "yarn", 8.0, 4096)
    n = 4096 * f / (2 * np.pi)
    assert np.array_equal(y[n >= 32], f[n >= 32]) and np.allclose(y[n <= 1], f[n <= 1] / 8)
    mid = (n > 1) & (n < 32)
    assert mid.any() and (y[mid] < f[mid]).all() and (y[mid] > f[mid] / 8).all() and g == 0.1 * np.log(8) + 1


@built
@pytest.mark.parametrize("kw", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=130), dict(base=0.0), dict(base=float("nan")),
                                dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("inf")),
                                dict(rotary_dim=2, scaling="ntk", factor=2.0), dict(scaling="yarn", factor=2.0),
                                dict(scaling="yarn", factor=2.0, original_len=10, beta_fast=1.0, beta_slow=1.0),
                                dict(scaling="yarn", factor=2.0, original_len=10, beta_slow=0.0)])
def test_frequency_refusals(kw):
    with pytest.raises((tm.TilemixError, ValueError)):
        tm.tilemix_rotary_frequencies(**{"rotary_dim": 64, "device": "cpu", **kw})
    with pytest.raises(ValueError):
        tm.tilemix_rotary_frequencies(64, scaling="cubic", device="cpu")
