"""GPU: decode over the paged cache with scores, values and queries far from 1."""

import numpy as np
import pytest
import torch

from gpu_util import log
from test_gpu_paged import FORMATS, PAIRS, _gen, _tm, _values

pytestmark = pytest.mark.gpu


def _cache_of(fmt, K, V, page):
    """K, V [L, d] (16 bits, CPU) written as the only sequence of a pool with one KV head: cache, table, lengths, and
    the float64 keys and values that the cache stands for."""
    tm = _tm()
    L, d = K.shape
    pages = -(-L // page)
    cache = tm.PagedCache.empty(pages, page, 1, d, FORMATS[fmt])
    table = torch.randperm(pages, generator=_gen(1)).to(torch.int32).view(1, pages)
    lens = torch.tensor([L], dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K[None, :, None].cuda(), V[None, :, None].cuda(), table.cuda(), lens)
    torch.cuda.synchronize()
    host = [None if t is None else t.cpu() for t in cache]
    k, v = (_values(host, op, fmt)[table[0].numpy(), 0].reshape(-1, d)[:L] for op in (0, 1))
    return cache, table.cuda(), lens, k, v


def _decode(cache, table, lens, Q, scale=None):
    """(O [Hq, d], lse [Hq]) as float64."""
    O, lse = _tm().tilemix_paged_decode(cache, Q.cuda(), table, lens, scale, return_lse=True)
    torch.cuda.synchronize()
    return O[0, 0].double().cpu().numpy(), lse[0].double().cpu().numpy()


# ------------------------------------------------------------------------------------ large scores

@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("L", [1, 3, 40, 300, 9000])
def test_large_scores(fmt, dtype, L):
    """Scores of 2^23 to 2^28 (log2 units), from ordinary FP16 numbers.  Two thirds of the keys equal the query up to a
    factor, the others are their negatives: the former have the same score, so equal weights, the latter's are 0, and
    O is the mean of the former's values.  Equal scores are equal to the last bit, whatever they were rounded to, so
    that what is left is the weights' pieces (2^-15 for a BF16 cache, 2^-22 for the others), sums of n terms and the
    normalizer (n 2^-24 each), a quotient and the output's rounding.  lse: d products and sums, the scale and its
    product with log2 e, and the last product, relative to the score."""
    d, page = 128, 64
    f = torch.finfo(FORMATS[dtype])
    for i, (q, v_gain) in enumerate([(300.0, 1.0), (1500.0, 1.0), (1500.0, 0.3), (2600.0, 37.0), (4000.0, 0.6), (7000.0, 1.0)]):
        sign = torch.ones(L, 1)
        sign[2::3] = -1
        K = (sign * 1500.0).expand(L, d).to(FORMATS[dtype])
        V = (torch.randn(L, d, generator=_gen(10 + i)) * v_gain).to(FORMATS[dtype])
        cache, table, lens, k, v = _cache_of(fmt, K, V, page)
        Q = torch.full((1, 1, 3, d), q).to(FORMATS[dtype])
        log(f"large scores {fmt}/{dtype} L {L} q {q}")
        O, lse = _decode(cache, table, lens, Q)
        heavy = sign[:, 0].numpy() > 0
        n = int(heavy.sum())
        want, mass = v[heavy].mean(0), np.abs(v[heavy]).mean(0)
        piece = 2.0 ** -15 if fmt == "bf16" else 2.0 ** -22
        v_max = 0.0 if fmt == "bf16" else np.abs(v).max()
        tol = f.eps / 2 * np.abs(want) + f.smallest_normal * f.eps + (piece + (2 * n + 4) * 2.0 ** -24) * mass + n * 2.0 ** -39 * v_max
        s = d ** -0.5 * (k[0] @ Q[0, 0, 0].double().numpy())
        for h in range(3):
            assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), (q, h)
            assert abs(lse[h] - (s + np.log(n))) <= (d + 8) * 2.0 ** -24 * s, (q, h)


# ------------------------------------------------------------- values of very different magnitudes

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("first", [0, 60])
@pytest.mark.parametrize("L,cut", [(64, 32), (160, 128), (320, 48), (9000, 4500), (9000, 8990)])
def test_values_of_zero_beside_large_ones(fmt, first, L, cut):
    """Tokens before `cut` have values 0 (first = 0) or around 2^-60, those behind it around 2^60, and the other way
    round; all keys are 0, so all scores are.  The cut lies between tiles of one wave, of several, and between
    workgroups.  Every token counts alike: lse = ln L, and O is the mean of the values.  Weights' pieces (2^-22) and
    sums (L 2^-24) as ever; lse: the normalizer's sum and the logarithm."""
    d, page = 64, 16
    f = torch.finfo(torch.bfloat16)
    for turn in (False, True):
        gain = torch.full((L, 1), 2.0 ** 60)
        gain[:cut] = 2.0 ** -first if first else 0.0
        V = (torch.randn(L, d, generator=_gen(30)) * (gain.flip(0) if turn else gain)).bfloat16()
        cache, table, lens, k, v = _cache_of(fmt, torch.zeros(L, d).bfloat16(), V, page)
        Q = torch.randn(1, 1, 2, d, generator=_gen(31)).bfloat16()
        log(f"values of zero beside large ones {fmt} 2^-{first} L {L} cut {cut} turned {turn}")
        O, lse = _decode(cache, table, lens, Q)
        want, mass = v.mean(0), np.abs(v).mean(0)
        tol = f.eps / 2 * np.abs(want) + (2.0 ** -22 + (2 * L + 4) * 2.0 ** -24) * mass + L * 2.0 ** -39 * np.abs(v).max()
        for h in range(2):
            assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), (turn, h)
            assert abs(lse[h] - np.log(L)) <= L * 2.0 ** -24 + 2.0 ** -21 * np.log(L), (turn, h)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("L", [5, 300, 5000])
@pytest.mark.parametrize("power", [-126, -120, -115, -110, -105, -100, -90, 100, 126])
def test_values_over_all_of_bf16(fmt, L, power):
    """BF16 values around 2^power, down to where the scales of their rows are subnormal, and no other ones.  Scores are
    exact (keys of one channel, +-1): weights are off by the exponent's argument and the exponent (2^-21 of scores up
    to 2), the pieces and sums; O by its rounding, to a multiple of 2^-133 at the bottom, and by one more in FP32."""
    d, page = 128, 32
    f = torch.finfo(torch.bfloat16)
    K = torch.zeros(L, d)
    K[:, 0] = torch.where(torch.arange(L) % 5 < 2, 1.0, -1.0)
    V = (torch.randn(L, d, generator=_gen(40)).clamp(-3, 3).double() * 2.0 ** (power - 1)).bfloat16()
    cache, table, lens, k, v = _cache_of(fmt, K.bfloat16(), V, page)
    Q = torch.zeros(1, 1, 2, d)
    Q[:, :, 0, 0], Q[:, :, 1, 0] = 1.0, -1.0
    log(f"values of 2^{power} {fmt} L {L}")
    O, lse = _decode(cache, table, lens, Q.bfloat16(), 0.75)
    for h, sign in ((0, 1.0), (1, -1.0)):
        s = 0.75 * sign * k[:, 0]
        p = np.exp(s)
        want, mass = p @ v / p.sum(), p @ np.abs(v) / p.sum()
        tol = (f.eps / 2 * np.abs(want) + 2.0 ** -133 / 2 + 2.0 ** -149 +
               (2.0 ** -20 + 2.0 ** -22 + (2 * L + 4) * 2.0 ** -24) * mass + L * 2.0 ** -39 * np.abs(v).max())
        assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), h
        assert abs(lse[h] - np.log(p.sum())) <= 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -21 * np.log(L), h


@pytest.mark.parametrize("fmt,power", [("fp16", p) for p in (-24, -20, -15, 0, 14)] +
                         [("bf16", p) for p in (-133, -130, -127, -120, -60, 60, 112)])
@pytest.mark.parametrize("L", [5, 300, 5000])
def test_values_over_all_of_16_bits(fmt, L, power):
    """The same for caches of 16 bits, subnormal values among them; BF16 up to 2^128 / L."""
    d, page = 128, 32
    f = torch.finfo(FORMATS[fmt])
    K = torch.zeros(L, d)
    K[:, 0] = torch.where(torch.arange(L) % 5 < 2, 1.0, -1.0)
    V = (torch.randn(L, d, generator=_gen(45)).clamp(-3, 3).double() * 2.0 ** (power - 1)).to(FORMATS[fmt])
    cache, table, lens, k, v = _cache_of(fmt, K.to(FORMATS[fmt]), V, page)
    Q = torch.zeros(1, 1, 2, d)
    Q[:, :, 0, 0], Q[:, :, 1, 0] = 1.0, -1.0
    log(f"values of 2^{power} {fmt} L {L}")
    O, lse = _decode(cache, table, lens, Q.to(FORMATS[fmt]), 0.75)
    v_max = np.abs(v).max() if fmt == "fp16" else 0.0
    for h, sign in ((0, 1.0), (1, -1.0)):
        s = 0.75 * sign * k[:, 0]
        p = np.exp(s)
        want, mass = p @ v / p.sum(), p @ np.abs(v) / p.sum()
        piece = 2.0 ** -16 if fmt == "bf16" else 2.0 ** -22
        tol = (f.eps / 2 * np.abs(want) + f.smallest_normal * f.eps / 2 + 2.0 ** -149 +
               (2.0 ** -20 + piece + (2 * L + 4) * 2.0 ** -24) * mass + L * 2.0 ** -39 * v_max)
        assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), h
        assert abs(lse[h] - np.log(p.sum())) <= 2.0 ** -20 + L * 2.0 ** -24 + 2.0 ** -21 * np.log(L), h


# ---------------------------------------------------------------------------------- small queries

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("power", [-128, -122, -112, -100, 100, 120])
def test_queries_over_all_of_bf16(fmt, power):
    """BF16 queries around 2^power against keys around 2^-power, so that scores are ordinary ones: off by
    (d + 8) 2^-24 of sum |q_c k_c|, as for queries near 1."""
    d, page, L = 64, 16, 90
    f = torch.finfo(torch.bfloat16)
    q_gain, k_gain = 2.0 ** power, 2.0 ** min(-power, 124)
    K = (torch.randn(L, d, generator=_gen(50)).clamp(-3, 3).double() * k_gain).bfloat16()
    V = torch.randn(L, d, generator=_gen(51)).bfloat16()
    cache, table, lens, k, v = _cache_of(fmt, K, V, page)
    Q = (torch.randn(1, 1, 3, d, generator=_gen(52)).double() * q_gain).bfloat16()
    log(f"queries of 2^{power} {fmt}")
    O, lse = _decode(cache, table, lens, Q, 0.5)
    for h in range(3):
        q = Q[0, 0, h].double().numpy()
        s = 0.5 * (k @ q)
        ds = (d + 8) * 2.0 ** -24 * 0.5 * (np.abs(k) @ np.abs(q)).max()
        p = np.exp(s - s.max())
        want, mass = p @ v / p.sum(), p @ np.abs(v) / p.sum()
        tol = f.eps / 2 * np.abs(want) + (2 * ds + 2.0 ** -20 + (2 * L + 4) * 2.0 ** -24) * mass + L * 2.0 ** -39 * np.abs(v).max()
        assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), h
        assert abs(lse[h] - (s.max() + np.log(p.sum()))) <= ds + L * 2.0 ** -24 + 2.0 ** -20, h


# ------------------------------------------------------------------------------ the weights' pieces

@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("d", [64, 128])
def test_small_sums_of_large_terms(fmt, dtype, d):
    """The last token's values cancel the sum of the others, as far as its format can: what is left of O is small, and
    so is its rounding, beside the weights' (2^-22 in two FP16 pieces, 2^-16 in two BF16 ones; one piece would be
    2^-12 or 2^-9 off).  Keys and queries are small whole numbers and row maxima the formats' tops, so that products are exact
    and scores are off by their scaling, log2 e and the exponent's argument only: 2^-24 each of |s| <= 8, a weight by twice
    that and the exponent, 2^-22; sums by n 2^-24."""
    n, page = 24, 16
    f = torch.finfo(FORMATS[dtype])
    top = {"int8": 127.0, "e4m3": 448.0}.get(fmt, 0.0)
    g = _gen(60)
    K = torch.randint(-2, 3, (n, d), generator=g).float()
    Q = torch.randint(-2, 3, (1, 1, 2, d), generator=g).float()
    if top:
        K[:, 0], Q[..., 0] = top, 0.0
    Q[0, 0, 1] = Q[0, 0, 0]
    q = Q[0, 0, 0]
    K[-1, 1:] = q[1:]                                                # the heaviest token
    if not top:
        K[-1, 0] = q[0]
    s = (K @ q).double()
    scale = 2.0 ** -int(np.ceil(np.log2(float(s.abs().max()) / 4.0)))
    p = torch.exp(scale * s)
    V = torch.randn(n, d, generator=g)
    V[-1] = 0
    V = V.to(FORMATS[dtype])
    v0 = _cache_of(fmt, K.to(FORMATS[dtype]), V, page)[4]           # as they are held
    V[-1] = torch.from_numpy(-(p.numpy() @ v0) / float(p[-1])).to(FORMATS[dtype])
    cache, table, lens, k, v = _cache_of(fmt, K.to(FORMATS[dtype]), V, page)
    assert np.array_equal(k, K.double().numpy())
    O, lse = _decode(cache, table, lens, Q.to(FORMATS[dtype]), scale)
    P = p.numpy() / float(p.sum())
    want, mass = P @ v, P @ np.abs(v)
    assert np.median(np.abs(want)) <= 2.0 ** -6 * np.median(mass)
    rel = 2 * 3 * 8 * 2.0 ** -24 + 2.0 ** -22 + (2.0 ** -16 if fmt == "bf16" else 2.0 ** -22) + (2 * n + 4) * 2.0 ** -24
    tol = f.eps / 2 * np.abs(want) + rel * mass + n * 2.0 ** -39 * np.abs(v).max()
    for h in range(2):
        log(f"small sums {fmt}/{dtype} d {d}: error/tolerance {np.max(np.abs(O[h] - want) / tol):.3f}, left {np.median(np.abs(want) / mass):.2g}")
        assert (np.abs(O[h] - want) <= tol * (1 + f.eps)).all(), h
