"""Oracle: a paged key/value cache - row quantisation, writing, reading back, one decode step
(test infrastructure only).

Plain float64 NumPy from the definitions: a row x with a = max |x| is held as codes
c = round(top x / a), half to even, on the whole numbers (top 127) or the E4M3 numbers (top 448), and
the float32 scale a / top; in MXFP4 the 32 channels of a block share 2^e, e the least integer >= -127 with all
magnitudes below 7 2^e, and a code is the E2M1 number nearest to x 2^-e, half to even; token t of sequence b lies in slot t % page of page table[b][t // page],
and a page id outside the pool names no page.

Pins: tests/test_oracle_paged.py.
"""

from __future__ import annotations

import numpy as np

TOP = {"int8": 127.0, "e4m3": 448.0}


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """The E4M3 number nearest to y (float64, |y| <= 448), half to even: 4 significant bits, spaced 2^-9 below
    2^-6."""
    _, e = np.frexp(y)
    step = np.exp2(np.maximum(e, -5) - 4.0)
    return np.rint(y / step) * step


def row_codes(x: np.ndarray, fmt: str):
    """(codes as float64 values [.., d], scale float32 [..]) of rows x [.., d]."""
    x = np.asarray(x, np.float64)
    a = np.max(np.abs(x), axis=-1, keepdims=True)      # NaN if the row holds one
    ok = np.isfinite(a) & (a > 0)
    with np.errstate(invalid="ignore", divide="ignore"):
        y = np.where(ok, TOP[fmt] * x / np.where(ok, a, 1.0), 0.0)
        scale = np.where(np.isfinite(a), a.astype(np.float32) / np.float32(TOP[fmt]), np.float32(np.nan))
    return (np.rint(y) if fmt == "int8" else round_e4m3(y)), scale[..., 0].astype(np.float32)


E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_e2m1(y: np.ndarray) -> np.ndarray:
    """The E2M1 number nearest to y (float64, |y| < 7), half to even: 2 significant bits, spaced 1/2 below 2."""
    _, e = np.frexp(y)
    step = np.exp2(np.maximum(e, 1) - 2.0)
    return np.rint(y / step) * step


def block_codes(x: np.ndarray):
    """(codes as float64 values [.., d] with the signs of x, exponent bytes uint8 [.., d / 32]) of rows x [.., d]."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    codes, byte = np.zeros_like(blocks), np.zeros(blocks.shape[:-1], np.uint8)
    for at in np.ndindex(byte.shape):
        a = np.max(np.abs(blocks[at]))                 # NaN if the block holds one
        if not np.isfinite(a):
            byte[at] = 255
            continue
        e = -127
        while a >= 7 * 2.0 ** e:
            e += 1
        codes[at] = np.copysign(round_e2m1(blocks[at] * 2.0 ** -e), blocks[at])
        byte[at] = e + 127
    return codes.reshape(x.shape), byte


def pack_e2m1(codes: np.ndarray) -> np.ndarray:
    """Bytes [.., d / 2] of E2M1 numbers [.., d]: sign, then the position in E2M1; the even channel in the low bits."""
    c = np.searchsorted(E2M1, np.abs(codes)) + 8 * np.signbit(codes)
    return (c[..., 0::2] + 16 * c[..., 1::2]).astype(np.uint8)


def mx_values(packed: np.ndarray, byte: np.ndarray) -> np.ndarray:
    """The float64 values [.., d] that bytes [.., d / 2] and exponent bytes [.., d / 32] stand for (255: NaN)."""
    c = np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], -1).astype(int)
    unit = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    return E2M1[c & 7] * np.where(c & 8, -1.0, 1.0) * np.repeat(unit, 32, -1)


def slot_of(table: np.ndarray, pages: int, page: int, b: int, t: int):
    """(page, slot) of token t of sequence b, or None."""
    if t < 0 or t >= table.shape[1] * page:
        return None
    p = int(table[b, t // page])
    return (p, t % page) if 0 <= p < pages else None


def new_tokens(seqlens, cu, B: int, length: int, total: int):
    """(sequence, packed row, token number) of every row that an append or gather deals with."""
    out = []
    for b in range(B):
        first, n = (b * length, length) if cu is None else (int(cu[b]), int(cu[b + 1]) - int(cu[b]))
        out += [(b, first + r, int(seqlens[b]) - n + r) for r in range(min(n, length))]
    return out


def attended(seqlens, table, pages: int, page: int, b: int, window: int):
    """(pages, slots) of the tokens that sequence b's query attends to."""
    n = min(max(int(seqlens[b]), 0), table.shape[1] * page)
    got = [slot_of(table, pages, page, b, t) for t in range(max(0, n - window) if window else 0, n)]
    got = [g for g in got if g is not None]
    return np.array([g[0] for g in got], int), np.array([g[1] for g in got], int)


def paged_decode(Q, K, V, seqlens, table, scale: float, window: int = 0):
    """O [B, Hq, d] and lse [B, Hq] in float64 for Q [B, Hq, d] and pools K, V [P, Hk, page, d] of values;
    and per head sum_j p_j |v_j| [B, Hq, d] and the largest scale sum_c |q_c k_jc| [B, Hq], which error bounds
    are made of."""
    B, Hq, d = Q.shape
    P, Hk, page, _ = K.shape
    O, mass = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    lse, reach = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    for b in range(B):
        ids, slots = attended(seqlens, table, P, page, b, window)
        if not len(ids):
            continue
        for h in range(Hk):
            k, v = K[ids, h, slots].astype(np.float64), V[ids, h, slots].astype(np.float64)
            for hq in range(h * (Hq // Hk), (h + 1) * (Hq // Hk)):
                q = Q[b, hq].astype(np.float64)
                s = scale * (k @ q)
                m = s.max()
                p = np.exp(s - m)
                z = p.sum()
                O[b, hq], mass[b, hq] = p @ v / z, p @ np.abs(v) / z
                lse[b, hq] = m + np.log(z)
                reach[b, hq] = scale * (np.abs(k) @ np.abs(q)).max()
    return O, lse, mass, reach
