"""GPU: the paged key/value cache - append and gather bit for bit, decode against float64."""

import numpy as np
import pytest
import torch

from gpu_util import log
from oracle.paged import TOP, new_tokens, paged_decode, row_codes, slot_of

pytestmark = pytest.mark.gpu

FORMATS = {"fp16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}
PAIRS = [("fp16", "fp16"), ("bf16", "bf16"), ("int8", "fp16"), ("int8", "bf16"), ("e4m3", "fp16"), ("e4m3", "bf16")]


def _tm():
    import paper_2608_17336_amd as tm
    return tm


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _bits(t):
    return t.cpu().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.dtype.itemsize])


def _random_pool(fmt, shape, seed):
    """A pool (CPU) of arbitrary bits, NaN patterns among them."""
    g = _gen(seed)
    P, H, page, d = shape
    size = FORMATS[fmt].itemsize
    K, V = (torch.randint(0, 256, (P, H, page, d * size), generator=g, dtype=torch.uint8).view(FORMATS[fmt]) for _ in "KV")
    dK, dV = (torch.randn(P, H, page, generator=g) for _ in "KV")
    return (K, V, dK, dV) if fmt in TOP else (K, V, None, None)


def _on_gpu(pool):
    return _tm().PagedCache(*[None if t is None else t.cuda() for t in pool])


def _write(pool, fmt, x, op, page, slot):
    """Oracle: row x [Hk, d] of operand op (0 K, 1 V) into (page, slot) of a CPU pool."""
    if fmt not in TOP:
        pool[op][page, :, slot] = x
        return
    codes, scale = row_codes(x.double().numpy(), fmt)
    codes = torch.from_numpy(codes)
    q = codes.to(torch.int8) if fmt == "int8" else (codes + 0.0).float().to(torch.float8_e4m3fn)
    pool[op].view(torch.uint8)[page, :, slot] = q.view(torch.uint8)
    pool[op + 2][page, :, slot] = torch.from_numpy(scale)


def _same_pool(got, want):
    for t, w, name in zip((got.K, got.V, got.dK, got.dV), want, ("K", "V", "dK", "dV")):
        if w is None:
            continue
        a, b = t.cpu(), w
        nan = torch.isnan(a.float()) & torch.isnan(b.float())       # a NaN scale has any payload
        minus0 = (a.float() == 0) & (b.float() == 0)                # codes of -0 and +0
        bad = (_bits(a) != _bits(b)) & ~nan & ~minus0
        assert not bad.any(), f"{name}: {int(bad.sum())} values differ, first at {bad.nonzero()[0].tolist()}"


def _table(B, per, pages, seed):
    return torch.randperm(pages, generator=_gen(seed))[: B * per].to(torch.int32).view(B, per)


def _rows(n, H, d, dtype, seed):
    x = torch.randn(n, H, d, generator=_gen(seed)) * torch.logspace(-3, 3, max(n, 1)).view(-1, 1, 1)[:n]
    return x.to(FORMATS[dtype])


# ------------------------------------------------------------------------- append and gather

@pytest.mark.parametrize("d,page,Hk", [(64, 16, 1), (64, 256, 3), (128, 64, 8), (128, 32, 2), (128, 16, 33)])
@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_append_then_gather_packed(fmt, dtype, d, page, Hk):
    """Ragged packed rows, written and read back bit for bit; nothing else changes."""
    tm = _tm()
    new = [0, 1, 2 * page + 3, page, 17]
    old = [5, 0, page - 2, 0, 3 * page + 1]
    B, per, pages = len(new), 6, 40
    lens = [o + n for o, n in zip(old, new)]
    cu = np.concatenate([[0], np.cumsum(new)])
    total = int(cu[-1]) + 4                                          # four rows that no sequence owns
    pool = _random_pool(fmt, (pages, Hk, page, d), d + page)
    table = _table(B, per, pages, 1)
    K, V = _rows(total, Hk, d, dtype, 2), _rows(total, Hk, d, dtype, 3)
    cache = _on_gpu(pool)
    t_gpu, l_gpu = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    cu_gpu = torch.tensor(cu, dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), t_gpu, l_gpu, cu_gpu, max(new))
    for b, r, t in new_tokens(lens, cu, B, max(new), total):
        p, s = slot_of(table.numpy(), pages, page, b, t)
        _write(pool, fmt, K[r], 0, p, s)
        _write(pool, fmt, V[r], 1, p, s)
    torch.cuda.synchronize()
    _same_pool(cache, pool)

    outK, outV = (torch.full((total, Hk, d), 7.0, dtype=FORMATS[dtype], device="cuda") for _ in "KV")
    tm.tilemix_paged_gather(cache, t_gpu, l_gpu, max(new), cu_gpu, K=outK, V=outV)
    for x, op, out in ((K, 0, outK), (V, 1, outV)):
        want = torch.full((total, Hk, d), 7.0, dtype=FORMATS[dtype])
        for b, r, t in new_tokens(lens, cu, B, max(new), total):
            p, s = slot_of(table.numpy(), pages, page, b, t)
            row = pool[op][p, :, s].float()
            want[r] = (row * pool[op + 2][p, :, s, None] if fmt in TOP else row).to(FORMATS[dtype])
        assert torch.equal(out.cpu(), want), ("KV"[op],)
        if fmt in TOP:   # at most half a step of the row from what was written
            x, got, n = x.double()[: int(cu[-1])], out.cpu().double()[: int(cu[-1])], int(cu[-1])
            a = x.abs().amax(-1, keepdim=True)
            half = a / 254 if fmt == "int8" else torch.maximum(x.abs() * 2.0 ** -4, a / 448 * 2.0 ** -10)
            tiny = torch.finfo(FORMATS[dtype])
            assert ((got - x).abs() <= half * (1 + 2.0 ** -20) + (got.abs() + half) * tiny.eps / 2 + tiny.tiny).all()


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("B,L,Hk,d", [(1, 1, 1, 64), (70, 1, 2, 128), (3, 5, 8, 128), (2, 130, 2, 64)])
def test_append_padded_and_strided(fmt, dtype, B, L, Hk, d):
    """[B, L, Hk, d] rows that are slices of a fused projection; pages that are slices of a tensor of K and
    V; a page table that is a slice; sequences that are shorter than L."""
    tm = _tm()
    page, per = 16, 10
    pages = B * per + 1
    both = torch.stack(_random_pool(fmt, (pages, Hk, page, d), 5)[:2], 1)
    scales = torch.randn(pages, 2, Hk, page, generator=_gen(6)) if fmt in TOP else None
    lens = [int(x) for x in torch.randint(0, per * page, (B,), generator=_gen(7))]
    lens[0] = min(L, 3)
    wide = torch.full((B, per + 2), -7, dtype=torch.int32)
    wide[:, :per] = _table(B, per, pages, 8)
    table = wide[:, :per]
    fused = _rows(B * L, 3 * Hk, d, dtype, 9).view(B, L, 3 * Hk, d)
    K, V = fused[:, :, Hk:2 * Hk], fused[:, :, 2 * Hk:]
    gb, gs, gf = both.cuda(), None if scales is None else scales.cuda(), fused.cuda()
    cache = tm.PagedCache(gb[:, 0], gb[:, 1], *((gs[:, 0], gs[:, 1]) if fmt in TOP else (None, None)))
    l_gpu, t_gpu = torch.tensor(lens, dtype=torch.int32).cuda(), wide.cuda()[:, :per]
    tm.tilemix_paged_append(cache, gf[:, :, Hk:2 * Hk], gf[:, :, 2 * Hk:], t_gpu, l_gpu)
    pool = [both[:, 0], both[:, 1]] + ([scales[:, 0], scales[:, 1]] if fmt in TOP else [None, None])
    for b, r, t in new_tokens(lens, None, B, L, B * L):
        at = slot_of(table.numpy(), pages, page, b, t)
        if at:
            _write(pool, fmt, K[b, r - b * L], 0, *at)
            _write(pool, fmt, V[b, r - b * L], 1, *at)
    torch.cuda.synchronize()
    _same_pool(cache, pool)
    gK, gV = tm.tilemix_paged_gather(cache, t_gpu, l_gpu, L, dtype=FORMATS[dtype])
    assert gK.shape == gV.shape == (B, L, Hk, d)
    short = L - lens[0]                                              # rows before the first token are zeros
    assert not gK[0, :short].any() and not gV[0, :short].any()
    if fmt not in TOP:
        assert torch.equal(gK.cpu()[0, short:], K[0, short:]) and torch.equal(gV.cpu()[0, short:], V[0, short:])


@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_append_rows_without_a_slot(fmt, dtype):
    """Missing pages, tokens past the page table, lengths below the new rows: nothing is written there, and
    reading gives zeros."""
    tm = _tm()
    page, per, pages, Hk, d = 16, 3, 12, 2, 128
    table = _table(4, per, pages, 11)
    table[0, 1], table[1, 0], table[2, 2] = -1, pages, 2 ** 31 - 1
    lens, new = [40, 20, 55, -5], [30, 20, 50, 6]                    # 55 > 48 slots; -5: all before the first
    cu = np.concatenate([[0], np.cumsum(new)])
    total = int(cu[-1])
    pool = _random_pool(fmt, (pages, Hk, page, d), 12)
    cache = _on_gpu(pool)
    K, V = _rows(total, Hk, d, dtype, 13), _rows(total, Hk, d, dtype, 14)
    args = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    cu_gpu = torch.tensor(cu, dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), *args, cu_gpu, 50)
    missing = []
    for b, r, t in new_tokens(lens, cu, 4, 50, total):
        at = slot_of(table.numpy(), pages, page, b, t)
        if at:
            _write(pool, fmt, K[r], 0, *at)
            _write(pool, fmt, V[r], 1, *at)
        else:
            missing.append(r)
    torch.cuda.synchronize()
    _same_pool(cache, pool)
    assert len(missing) > 30
    gK, gV = tm.tilemix_paged_gather(cache, *args, 50, cu_gpu, total, dtype=FORMATS[dtype])
    assert not gK[missing].any() and not gV[missing].any()
    kept = [r for r in range(total) if r not in missing]
    assert gK[kept].any(-1).any(-1).all()


@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_rows_of_many_sequences(fmt, dtype):
    """More sequences than lanes of a wave, most with few rows or none; the same through a call that takes the first
    40 rows of each at most."""
    tm = _tm()
    B, Hk, d, page, per = 150, 2, 64, 16, 7
    new = [(0, 0, 1, 7, 100, 33)[b * b % 6] for b in range(B)]
    lens = [n + b % 5 for b, n in enumerate(new)]
    cu = np.concatenate([[0], np.cumsum(new)])
    total, pages = int(cu[-1]), B * per
    table = _table(B, per, pages, 40)
    K, V = _rows(total, Hk, d, dtype, 41), _rows(total, Hk, d, dtype, 42)
    t_gpu, l_gpu, cu_gpu = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor(cu, dtype=torch.int32).cuda()
    for longest in (100, 40):
        pool = _random_pool(fmt, (pages, Hk, page, d), 43)
        cache = _on_gpu(pool)
        tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), t_gpu, l_gpu, cu_gpu, longest)
        rows = new_tokens(lens, cu, B, longest, total)
        for b, r, t in rows:
            at = slot_of(table.numpy(), pages, page, b, t)
            _write(pool, fmt, K[r], 0, *at)
            _write(pool, fmt, V[r], 1, *at)
        torch.cuda.synchronize()
        _same_pool(cache, pool)
        out = [torch.full((total, Hk, d), 7.0, dtype=FORMATS[dtype], device="cuda") for _ in "KV"]
        tm.tilemix_paged_gather(cache, t_gpu, l_gpu, longest, cu_gpu, K=out[0], V=out[1])
        for op in (0, 1):
            want = torch.full((total, Hk, d), 7.0, dtype=FORMATS[dtype])
            for b, r, t in rows:
                p, s = slot_of(table.numpy(), pages, page, b, t)
                row = pool[op][p, :, s].float()
                want[r] = (row * pool[op + 2][p, :, s, None] if fmt in TOP else row).to(FORMATS[dtype])
            assert torch.equal(out[op].cpu(), want)


def test_rows_of_broken_offsets():
    """cu_seqlens that step back or point outside the rows: no row beyond `total` is read or written."""
    tm = _tm()
    Hk, d, page, total = 2, 64, 16, 20
    cache = tm.PagedCache.empty(8, page, Hk, d, torch.float16)
    cache.K.zero_(), cache.V.zero_()
    table = torch.arange(8, dtype=torch.int32).view(4, 2).cuda()
    lens = torch.tensor([30, 30, 30, 30], dtype=torch.int32).cuda()
    cu = torch.tensor([-5, 12, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    buf = torch.full((total + 40, Hk, d), 3.0, dtype=torch.float16, device="cuda")
    tm.tilemix_paged_append(cache, buf[:total], buf[:total], table, lens, cu, 2 ** 20)
    tm.tilemix_paged_gather(cache, table, lens, 2 ** 20, cu, K=buf[:total], V=buf[:total].clone())
    torch.cuda.synchronize()
    assert (buf[total:] == 3.0).all()
    for b, n in enumerate((12, 0, 17, 0)):                           # at most rows 0 .. 11, none, rows 3 .. 19, none
        held = cache.K[2 * b:2 * b + 2].transpose(1, 2).reshape(2 * page, -1)
        assert ((held[30 - n:30] == 3.0) | (held[30 - n:30] == 0.0)).all() and not held[:30 - n].any() and not held[30:].any()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_append_special_rows(fmt, dtype, d):
    """Rows of zeros, subnormals, the largest values, ties (x = a / 2), infinities and NaN."""
    tm = _tm()
    f = torch.finfo(FORMATS[dtype])
    rows = torch.randn(16, 1, d, generator=_gen(20))
    rows[0] = 0
    rows[1] = 0
    rows[1, 0, 3] = f.smallest_normal * 2.0 ** -7                    # one subnormal value
    rows[2] *= f.smallest_normal                                     # around the smallest normal one
    rows[3] = rows[3].sign() * f.max
    rows[4] = torch.linspace(-f.max, f.max, d)                       # (BF16: its steps overflow, to NaN)
    rows[5] = torch.where(rows[5] > 0, 1.0, 0.5)
    rows[6] = torch.linspace(-127, 127, d)
    rows[7, 0, 1] = float("inf")
    rows[8, 0, d - 1] = -float("inf")
    rows[9, 0, 5] = float("nan")
    rows[10] = float("nan")
    rows[11] = -0.0
    rows[12] = torch.arange(d) * f.smallest_normal * f.eps           # subnormals only
    rows = rows.to(FORMATS[dtype])
    pool = _random_pool(fmt, (1, 1, 16, d), 21)
    cache = _on_gpu(pool)
    table, lens = torch.zeros(1, 1, dtype=torch.int32).cuda(), torch.tensor([16], dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, rows[None].cuda(), rows[None].cuda(), table, lens)
    for t in range(16):
        _write(pool, fmt, rows[t], 0, 0, t)
        _write(pool, fmt, rows[t], 1, 0, t)
    torch.cuda.synchronize()
    _same_pool(cache, pool)
    K, V = tm.tilemix_paged_gather(cache, table, lens, 16, dtype=FORMATS[dtype])
    K = K[0, :, 0].float().cpu()
    finite = torch.isfinite(rows).all(-1).all(-1)
    assert not finite[7:11].any() and finite[:4].all() and finite[11:].all()
    assert torch.isnan(K[~finite]).all() and not torch.isnan(K[finite]).any()
    assert not K[0].any() and not K[11].any()
    assert torch.equal(K[3], rows[3, 0].float())


def test_every_e4m3_and_int8_code():
    """Rows that hold every multiple of a's 1 / 2048: codes and values against the oracle."""
    tm = _tm()
    x = torch.cat([torch.arange(0, 2049), -torch.arange(0, 2047)]).float().view(32, 1, 128) / 1024
    x[:, :, 0] = 2.0 * torch.linspace(1, 1.999, 32).view(32, 1)     # a of 32 mantissas
    x = x.half()
    for fmt in TOP:
        pool = _random_pool(fmt, (2, 1, 16, 128), 22)
        cache = _on_gpu(pool)
        table, lens = torch.tensor([[1, 0]], dtype=torch.int32).cuda(), torch.tensor([32], dtype=torch.int32).cuda()
        tm.tilemix_paged_append(cache, x[None].cuda(), x[None].cuda(), table, lens)
        for t in range(32):
            _write(pool, fmt, x[t], 0, 1 - t // 16, t % 16)
            _write(pool, fmt, x[t], 1, 1 - t // 16, t % 16)
        torch.cuda.synchronize()
        _same_pool(cache, pool)


# ------------------------------------------------------------------------------------ decode

def _values(pool, op, fmt):
    """Float64 values of a CPU pool's operand; slots that a call must not use may hold NaN."""
    x = pool[op].double()
    return (x * pool[op + 2][..., None].double() if fmt in TOP else x).numpy()


def _cached_pool(fmt, shape, seed, gain=1.0):
    """A pool (CPU) of finite rows."""
    P, H, page, d = shape
    out = [None] * 4
    for op in (0, 1):
        x = torch.randn(shape, generator=_gen(seed + op)) * gain
        if fmt in TOP:
            codes, scale = row_codes(x.half().double().numpy(), fmt)
            codes = torch.from_numpy(codes)
            out[op] = codes.to(torch.int8) if fmt == "int8" else codes.float().to(torch.float8_e4m3fn)
            out[op + 2] = torch.from_numpy(scale)
        else:
            out[op] = x.to(FORMATS[fmt])
    return out


def _poison(pool, fmt, used):
    """Fill every slot outside ``used`` (bool [P, page]) with NaN (INT8 codes: with NaN scales)."""
    for op in (0, 1):
        if fmt == "int8":
            pool[op].masked_fill_(~used[:, None, :, None], -128)
        else:
            bad = torch.tensor(float("nan")).to(FORMATS[fmt])
            flat = pool[op].view(torch.uint8 if fmt == "e4m3" else torch.int16)
            flat.masked_fill_(~used[:, None, :, None], int(bad.view(flat.dtype)))
        if fmt in TOP:
            pool[op + 2].masked_fill_(~used[:, None, :], float("nan"))


def _check_decode(name, O, lse, want, dtype, n, v_max=0.0):
    """O: half a step of its type, and FP32 arithmetic: a score is off by at most (d + 8) 2^-24 reach (products and
    sums of d terms, the scale, log2 e) and 2^-22 |s| (the exponent's argument), a weight by twice the largest of these
    relative to the others, the weights' 16-bit pieces by 2^-15 (two pieces of 8 bits) and a sum of n terms by
    n 2^-24; these act on sum p |v|.  lse: the same without the pieces.
    v_max: the largest |v|, where weights are held in pieces of FP16 (all caches but BF16).  A weight
    w = 2^15 p dV / 2^e <= 2^15, with 2^e <= 2 max dV and z >= 1, is split into hi = RN16(w) and
    lo = RN16(w - hi) (the difference is exact): off by at most 2^-22 w (within 2^-15 above) or half
    the step of FP16's subnormals, 2^-25.  The n terms of the latter add n 2^-25 2^-15 2^e max |code| <=
    n 2^-39 v_max to O, whatever the weights: it shows where the heavy tokens' codes are 0."""
    wO, wl, mass, reach = want
    d = wO.shape[-1]
    f = torch.finfo(FORMATS[dtype])
    O, lse = O.double().cpu().numpy().reshape(wO.shape), lse.double().cpu().numpy()
    ds = (d + 8) * 2.0 ** -24 * reach + 2.0 ** -22 * np.maximum(np.where(np.isfinite(wl), np.abs(wl), 0), reach)
    rel = np.exp(2 * ds) - 1 + 2.0 ** -15 + n * 2.0 ** -24
    tol = f.eps / 2 * np.abs(wO) + f.smallest_normal * f.eps + (rel[..., None] * mass + n * 2.0 ** -39 * v_max) * (1 + f.eps)
    err = np.abs(O - wO)
    seen = np.isfinite(wl)
    l_tol = ds + n * 2.0 ** -24 + 2.0 ** -22 * (1 + np.abs(np.where(seen, wl, 0)))
    l_err = np.abs(np.where(seen, lse - np.where(seen, wl, 0), 0))
    log(f"decode {name}: O error/tolerance {np.nanmax(err / tol):.3f}, lse {np.max(l_err / l_tol):.3f}")
    assert np.isfinite(O).all() and (err <= tol).all(), name
    assert (np.isneginf(lse) == ~seen).all() and (l_err <= l_tol).all(), name
    # In the norm the errors of FP32 arithmetic do not add up: what is left is the output's rounding.
    norm = np.linalg.norm(wO)
    if norm:
        kappa = np.linalg.norm(mass) / norm
        assert np.linalg.norm(O - wO) <= norm * (f.eps / 2 + 2.0 ** -15 * kappa) + np.sqrt(wO.size) * f.smallest_normal * f.eps, name


def _v_max(V, fmt):
    return 0.0 if fmt == "bf16" else float(np.abs(V).max())


def _decode_case(fmt, dtype, Hq, Hk, d, page, lens, window=0, seed=0, holes=(), gain=1.0, q_gain=1.0, scale=None, per=None):
    tm = _tm()
    B = len(lens)
    per = per or max(1, max(-(-x // page) for x in lens))
    pages = B * per + 2
    table = _table(B, per, pages, seed + 30)
    for b, e, x in holes:
        table[b, e] = x
    pool = _cached_pool(fmt, (pages, Hk, page, d), seed + 31, gain)
    used = torch.zeros(pages, page, dtype=torch.bool)
    for b, L in enumerate(lens):
        for t in range(max(0, L - window) if window else 0, L):
            at = slot_of(table.numpy(), pages, page, b, t)
            if at:
                used[at] = True
    _poison(pool, fmt, used)
    for b, L in enumerate(lens):                                    # page ids past a length mean nothing
        table[b, -(-max(L, 0) // page):] = 2 ** 31 - 1 if b % 2 else -1
    Q = (torch.randn(B, 1, Hq, d, generator=_gen(seed + 40)) * q_gain).to(FORMATS[dtype])
    scale = scale or d ** -0.5
    cache = _on_gpu(pool)
    args = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    name = f"{fmt}/{dtype} {Hq}/{Hk} d{d} page {page} lens {lens[:6]} window {window}"
    log(f"decode {name}: start")
    O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), *args, scale, window=window, return_lse=True)
    torch.cuda.synchronize()
    K, V = (np.where(used.numpy()[:, None, :, None], _values(pool, op, fmt), 0.0) for op in (0, 1))
    want = paged_decode(Q.double().numpy()[:, 0], K, V, lens, table.numpy(), scale, window)
    _check_decode(name, O, lse, want, dtype, max(lens), _v_max(V, fmt))
    again = tm.tilemix_paged_decode(cache, Q.cuda(), *args, scale, window=window)
    torch.cuda.synchronize()
    assert torch.equal(_bits(again), _bits(O)), "the same call twice"


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("Hq,Hk,d,page", [(2, 2, 64, 16), (8, 1, 128, 64), (6, 2, 64, 32), (7, 1, 128, 16),
                                          (16, 1, 128, 256), (33, 3, 64, 128)])
def test_decode_lengths(fmt, dtype, Hq, Hk, d, page):
    """Lengths from none to several tiles: either side of slabs, tiles and pages."""
    _decode_case(fmt, dtype, Hq, Hk, d, page, [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 130, 255, 257, 300])


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("Hq,Hk", [(17, 1), (32, 1), (40, 2), (100, 1)])
def test_decode_large_groups(fmt, dtype, Hq, Hk):
    """More query heads per KV head than one block of 16."""
    _decode_case(fmt, dtype, Hq, Hk, 128, 32, [500, 3, 0, 77], seed=100)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("lens,Hq,Hk,d,page", [([5000], 8, 2, 128, 16), ([9001, 1], 4, 1, 64, 256), ([4096, 17, 2500], 8, 2, 64, 64)])
def test_decode_long(fmt, dtype, lens, Hq, Hk, d, page):
    """Caches that are split over workgroups."""
    _decode_case(fmt, dtype, Hq, Hk, d, page, lens, seed=200)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("Hq,Hk,d,long", [(2, 2, 64, 700), (6, 1, 128, 700), (128, 1, 64, 1100), (96, 2, 128, 1100)])
def test_decode_many_sequences(fmt, dtype, Hq, Hk, d, long):
    """More sequences than lanes of a wave, with empty ones at both ends; few and many beside the workgroups that
    run at once, so that a long sequence is cut, and a workgroup has parts of several."""
    lens = [(0, 3, 37, 150, 1, 64)[b * b % 6] for b in range(150)]
    lens[7] = lens[130] = long
    lens[149] = 0
    _decode_case(fmt, dtype, Hq, Hk, d, 16, lens, seed=1500)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("Hq,B,slots", [(4, 3, 480), (4, 3, 512), (4, 3, 544), (64, 64, 992), (64, 64, 1024), (64, 64, 1056),
                                        (128, 140, 256)])
def test_decode_capacities(fmt, dtype, Hq, B, slots):
    """Page tables of 15 to 17 and 31 to 33 tiles of 32 keys, full and empty sequences, one or several a workgroup."""
    lens = [slots, slots - 1, 0, 1] + [(b * 41 + 5) % 170 for b in range(4, B)]
    _decode_case(fmt, dtype, Hq, 1, 64, 32, lens[:B], seed=1600, per=slots // 32)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("B,per", [(100, 17), (250, 9)])
def test_decode_alike_lengths_in_long_page_tables(fmt, dtype, B, per):
    """Nearly equal sequences, as many as the workgroups that run at once or twice as many."""
    _decode_case(fmt, dtype, 128, 1, 64, 128, [300 - b % 7 for b in range(B - 1)] + [0], seed=1800, per=per)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("lens", [[65900, 0, 1, 100], [22000, 23000, 21100]])
def test_decode_of_a_large_batch(fmt, dtype, lens):
    """Caches larger than 2^27 bytes.  Few pages, each named many times (a prefix that sequences share)."""
    tm = _tm()
    d, page, pages = 128, 64, 20
    Hk = 8 if fmt in TOP else 4
    Hq = 2 * Hk
    assert sum(lens) * 2 * Hk * d * FORMATS[fmt].itemsize > 2 ** 27
    pool = _cached_pool(fmt, (pages, Hk, page, d), 1700)
    table = torch.randint(0, pages, (len(lens), -(-max(lens) // page)), generator=_gen(1701)).to(torch.int32)
    Q = torch.randn(len(lens), 1, Hq, d, generator=_gen(1702)).to(FORMATS[dtype])
    log(f"decode of a large batch {fmt}/{dtype} {lens}: start")
    O, lse = tm.tilemix_paged_decode(_on_gpu(pool), Q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), return_lse=True)
    torch.cuda.synchronize()
    # Equal tokens count alike: the oracle's softmax over a token per (page, slot), weighted by how often it occurs.
    K, V = _values(pool, 0, fmt), _values(pool, 1, fmt)
    times = np.zeros((len(lens), pages, page))
    for b, L in enumerate(lens):
        for t in range(L):
            times[b, int(table[b, t // page]), t % page] += 1
    q = Q.double().numpy()[:, 0]
    want = [np.zeros((len(lens), Hq, d)), np.full((len(lens), Hq), -np.inf), np.zeros((len(lens), Hq, d)), np.zeros((len(lens), Hq))]
    for b, hq in np.ndindex(len(lens), Hq):
        if not lens[b]:
            continue
        k, v = K[:, hq // 2].reshape(-1, d), V[:, hq // 2].reshape(-1, d)
        s = d ** -0.5 * (k @ q[b, hq])
        m = s.max()
        w = times[b].ravel() * np.exp(s - m)
        z = w.sum()
        want[0][b, hq], want[1][b, hq], want[2][b, hq] = w @ v / z, m + np.log(z), w @ np.abs(v) / z
        want[3][b, hq] = d ** -0.5 * (np.abs(k) @ np.abs(q[b, hq])).max()
    _check_decode(f"large batch {fmt}/{dtype}", O, lse, want, dtype, max(lens), _v_max(V, fmt))


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("window", [1, 16, 50, 64, 1000])
def test_decode_window(fmt, dtype, window):
    """The last tokens only; the pages before them are given back (-1)."""
    lens, page = [0, 1, 49, 50, 51, 64, 200, 1313], 16
    holes = [(b, e, -1) for b, L in enumerate(lens) for e in range(max(0, L - window) // page)]
    _decode_case(fmt, dtype, 8, 2, 128, page, lens, window=window, seed=300, holes=holes)
    _decode_case(fmt, dtype, 6, 3, 64, 128, lens, window=window, seed=301)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_decode_missing_pages(fmt, dtype, page):
    """Tokens without a page are left out; a sequence without any page gets 0."""
    lens = [3 * page, 5 * page - 3, 2 * page]
    holes = [(0, 1, -1), (1, 0, 2 ** 30), (1, 3, -2 ** 31), (2, 0, -1), (2, 1, 10 ** 6)]
    _decode_case(fmt, dtype, 8, 2, 128, page, lens, seed=400, holes=holes)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_decode_sharp_scores(fmt, dtype):
    """Scores of some hundreds (one token takes all the weight) and of nearly nothing (all alike)."""
    _decode_case(fmt, dtype, 8, 2, 128, 64, [700, 129], seed=500, q_gain=60.0)
    _decode_case(fmt, dtype, 8, 2, 128, 64, [700, 129], seed=501, q_gain=2.0 ** -10)


@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_decode_values_of_many_magnitudes(fmt, dtype):
    """A token with most of the weight and values near 0 beside tokens of little weight and ordinary values, in
    either order: the small contributions are not lost."""
    tm = _tm()
    d, page, L = 128, 64, 300
    for sink in (0, L - 1):
        pool = _cached_pool(fmt, (5, 1, page, d), 600)
        K = torch.zeros(5 * page, d)
        V = torch.randn(5 * page, d, generator=_gen(601))
        K[sink], V[sink] = 1.0, V[sink] * 2.0 ** -12
        cache = tm.PagedCache(*[torch.zeros_like(t).cuda() if t is not None else None for t in pool])
        table = torch.arange(5, dtype=torch.int32).view(1, 5).cuda()
        lens = torch.tensor([L], dtype=torch.int32).cuda()
        tm.tilemix_paged_append(cache, K[None, :L, None].to(FORMATS[dtype]).cuda(), V[None, :L, None].to(FORMATS[dtype]).cuda(),
                                table, lens)
        Q = torch.full((1, 1, 1, d), 13.0 / d ** 0.5).to(FORMATS[dtype])     # the sink's score: 13
        O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, return_lse=True)
        torch.cuda.synchronize()
        host = [None if t is None else t.cpu() for t in (cache.K, cache.V, cache.dK, cache.dV)]
        want = paged_decode(Q.double().numpy()[:, 0], _values(host, 0, fmt), _values(host, 1, fmt), [L], table.cpu().numpy(),
                            d ** -0.5)
        _check_decode(f"sink at {sink} {fmt}/{dtype}", O, lse, want, dtype, L, _v_max(_values(host, 1, fmt), fmt))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_decode_bf16_range(fmt):
    """Rows and queries beyond FP16's range: 2^60 and 2^-60."""
    tm = _tm()
    d, page, L = 64, 16, 90
    for gk, gv, gq in ((2.0 ** 60, 2.0 ** -60, 2.0 ** -60), (2.0 ** -60, 2.0 ** 60, 2.0 ** 60)):
        K = (torch.randn(1, L, 1, d, generator=_gen(700)) * gk).bfloat16()
        V = (torch.randn(1, L, 1, d, generator=_gen(701)) * gv).bfloat16()
        V[:, ::3] *= 2.0 ** -20
        Q = (torch.randn(1, 1, 3, d, generator=_gen(702)) * gq).bfloat16()
        cache = tm.PagedCache.empty(6, page, 1, d, FORMATS[fmt])
        table = torch.arange(6, dtype=torch.int32).view(1, 6).cuda()
        lens = torch.tensor([L], dtype=torch.int32).cuda()
        tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), table, lens)
        O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, return_lse=True)
        torch.cuda.synchronize()
        host = [t.cpu() for t in (cache.K, cache.V, cache.dK, cache.dV)]
        k, v = (np.nan_to_num(_values(host, op, fmt)) for op in (0, 1))
        want = paged_decode(Q.double().numpy()[:, 0], k, v, [L], table.cpu().numpy(), d ** -0.5)
        _check_decode(f"range {gk:g} {fmt}", O, lse, want, "bf16", L, _v_max(v, fmt))


@pytest.mark.parametrize("fmt,dtype", PAIRS)
def test_decode_nan_stays_in_its_sequence(fmt, dtype):
    """A NaN in one sequence's keys reaches that sequence's heads and nobody else."""
    tm = _tm()
    d, page = 128, 16
    pool = _cached_pool(fmt, (12, 2, page, d), 800)
    table = _table(3, 4, 12, 801)
    cache = _on_gpu(pool)
    lens = torch.tensor([60, 60, 60], dtype=torch.int32).cuda()
    Q = torch.randn(3, 1, 4, d, generator=_gen(802)).to(FORMATS[dtype]).cuda()
    before = tm.tilemix_paged_decode(cache, Q, table.cuda(), lens)
    bad = torch.full((3, 1, 2, d), 1.0).to(FORMATS[dtype])
    bad[1, 0, 1, 7] = float("nan")
    one = table.clone()
    one[0], one[2] = -1, -1                                          # only sequence 1 is written
    tm.tilemix_paged_append(cache, bad.cuda(), bad.cuda(), one.cuda(), lens)
    after = tm.tilemix_paged_decode(cache, Q, table.cuda(), lens)
    assert torch.isnan(after[1, 0, 2:]).any(-1).all() and not torch.isnan(after[1, 0, :2]).any()
    for b in (0, 2):
        assert torch.equal(_bits(after[b]), _bits(before[b]))


@pytest.mark.parametrize("fmt", ["fp16", "bf16"])
def test_decode_infinity_stays_in_its_channel(fmt):
    """An infinite value of a 16-bit cache reaches its channel of its sequence's heads, and nothing else."""
    tm = _tm()
    d, page = 128, 16
    pool = _cached_pool(fmt, (12, 2, page, d), 820)
    table = _table(3, 4, 12, 821)
    lens = torch.tensor([60, 60, 60], dtype=torch.int32).cuda()
    Q = torch.randn(3, 1, 4, d, generator=_gen(822)).to(FORMATS[fmt]).cuda()
    before = tm.tilemix_paged_decode(_on_gpu(pool), Q, table.cuda(), lens)
    pool[1][int(table[1, 2]), 1, 5, 9] = float("inf")                # token 37 of sequence 1, KV head 1, channel 9
    after = tm.tilemix_paged_decode(_on_gpu(pool), Q, table.cuda(), lens)
    hit = torch.zeros_like(before, dtype=torch.bool)
    hit[1, 0, 2:, 9] = True
    assert not torch.isfinite(after[hit]).any()
    assert torch.equal(_bits(after[~hit]), _bits(before[~hit]))


def test_decode_strided_queries_and_given_outputs():
    tm = _tm()
    d, page, B, Hq, Hk = 128, 16, 5, 8, 2
    pool = _cached_pool("int8", (20, Hk, page, d), 900)
    cache, table = _on_gpu(pool), _table(B, 4, 20, 901).cuda()
    lens = torch.tensor([64, 1, 0, 33, 16], dtype=torch.int32).cuda()
    fused = torch.randn(B, 1, Hq + 2 * Hk, d, generator=_gen(902)).half().cuda()
    Q = fused[:, :, :Hq]
    want = tm.tilemix_paged_decode(cache, Q.contiguous(), table, lens)
    O, lse = torch.full_like(want, 9.0), torch.full((B, Hq), 9.0, device="cuda")
    need = tm.tilemix_paged_decode_workspace_size(cache, table, lens, Hq)
    got, got_lse = tm.tilemix_paged_decode(cache, Q, table, lens, O=O, lse=lse, return_lse=True,
                                           workspace=torch.empty(need + 256, dtype=torch.uint8, device="cuda"))
    assert got is O and got_lse is lse
    assert torch.equal(_bits(O), _bits(want)) and not O[2].any()
    assert torch.isneginf(lse[2]).all() and torch.isfinite(lse[[0, 1, 3, 4]]).all()
    one = tm.tilemix_paged_decode(cache, Q[:1].expand(B, 1, Hq, d), table, lens)      # one query for all
    ref = tm.tilemix_paged_decode(cache, Q[:1].expand(B, 1, Hq, d).contiguous(), table, lens)
    assert torch.equal(_bits(one), _bits(ref))


def test_offsets_past_32_bits():
    """A pool whose pages lie beyond 2^32 bytes and 2^31 elements, read and written at its end."""
    tm = _tm()
    page, Hk, d = 256, 8, 128
    pages = 2 ** 31 // (page * Hk * d) + 20
    for fmt, dtype in (("fp16", "fp16"), ("int8", "bf16")):
        shape = (pages, Hk, page, d)
        K, V = (torch.empty(shape, dtype=FORMATS[fmt], device="cuda") for _ in "KV")
        if fmt == "int8":   # far apart, too: every second page of twice the pages
            K, V = (torch.empty((2 * pages, *shape[1:]), dtype=torch.int8, device="cuda")[::2] for _ in "KV")
            cache = tm.PagedCache(K, V, *(torch.empty(shape[:3], device="cuda") for _ in "KV"))
        else:
            cache = tm.PagedCache(K, V)
        table = torch.tensor([[pages - 1, 0, pages - 7], [1, pages - 2, pages - 3]], dtype=torch.int32).cuda()
        lens = torch.tensor([600, 513], dtype=torch.int32).cuda()
        cu = torch.tensor([0, 600, 1113], dtype=torch.int32).cuda()
        x, y = (_rows(1113, Hk, d, dtype, 950 + i).cuda() for i in range(2))
        x, y = x.clamp(-4, 4), y.clamp(-4, 4)
        tm.tilemix_paged_append(cache, x, y, table, lens, cu, 600)
        gK, gV = tm.tilemix_paged_gather(cache, table, lens, 600, cu, 1113, dtype=FORMATS[dtype])
        if fmt == "fp16":
            assert torch.equal(gK, x) and torch.equal(gV, y)
        # the same rows in a small pool
        small = tm.PagedCache.empty(6, page, Hk, d, FORMATS[fmt])
        st = torch.arange(6, dtype=torch.int32).view(2, 3).cuda()
        tm.tilemix_paged_append(small, x, y, st, lens, cu, 600)
        sK, sV = tm.tilemix_paged_gather(small, st, lens, 600, cu, 1113, dtype=FORMATS[dtype])
        assert torch.equal(gK, sK) and torch.equal(gV, sV)
        Q = torch.randn(2, 1, 16, d, generator=_gen(960)).to(FORMATS[dtype]).cuda()
        assert torch.equal(_bits(tm.tilemix_paged_decode(cache, Q, table, lens)), _bits(tm.tilemix_paged_decode(small, Q, st, lens)))
        del K, V, cache


# ------------------------------------------------------------------------------- as they are used

def _words(p):
    tm = _tm()
    return torch.from_numpy(tm.tilemix_route_template(p, tm.Template("zero")).view(np.int64)).cuda()


@pytest.mark.parametrize("fmt", ["fp16", "int8", "e4m3"])
def test_prefill_append_decode_and_chunked_prefill(fmt):
    """A prompt through tilemix_prefill and into the cache, steps of append and decode, then the next
    turn's rows against the prefix that is read back, through tilemix_prefill_varlen."""
    tm = _tm()
    Hq, Hk, d, page, L, steps, turn = 8, 2, 128, 64, 333, 5, 70
    g = _gen(1000)
    n = L + steps + turn
    q, k, v = (torch.randn(1, n, H, d, generator=g).half().cuda() for H in (Hq, Hk, Hk))
    cache = tm.PagedCache.empty(12, page, Hk, d, FORMATS[fmt])
    table = _table(1, 8, 12, 1001).cuda()
    lens = torch.tensor([L], dtype=torch.int32).cuda()
    p = tm.Params(1, Hq, Hk, L, L, d, 128, 64, 1, True, 0.0, False, 0)
    tm.tilemix_prefill(q[:, :L], k[:, :L], v[:, :L], _words(p), 1, route_hint=0)
    tm.tilemix_paged_append(cache, k[:, :L], v[:, :L], table, lens)
    outs = []
    for t in range(L, L + steps):
        lens += 1
        tm.tilemix_paged_append(cache, k[:, t:t + 1], v[:, t:t + 1], table, lens)
        outs.append(tm.tilemix_paged_decode(cache, q[:, t:t + 1], table, lens, return_lse=True))
    lens += turn
    tm.tilemix_paged_append(cache, k[:, -turn:], v[:, -turn:], table, lens)
    cu_k = torch.tensor([0, n], dtype=torch.int32).cuda()
    cu_q = torch.tensor([0, turn], dtype=torch.int32).cuda()
    gk, gv = tm.tilemix_paged_gather(cache, table, lens, n, cu_k, n)
    p = tm.Params(1, Hq, Hk, turn, n, d, 128, 64, 1, True, 0.0, False, 0)
    chunk = tm.tilemix_prefill_varlen(q[0, -turn:].contiguous(), gk, gv, cu_q, cu_k, turn, n, _words(p)[0].transpose(0, 1).contiguous(),
                                      1, route_hint=0)
    torch.cuda.synchronize()
    host = [None if t is None else t.cpu() for t in (cache.K, cache.V, cache.dK, cache.dV)]
    K, V = (np.nan_to_num(_values(host, op, fmt)) for op in (0, 1))
    for i, (O, lse) in enumerate(outs):
        want = paged_decode(q[:, L + i].double().cpu().numpy(), K, V, [L + i + 1], table.cpu().numpy(), d ** -0.5)
        _check_decode(f"step {i} {fmt}", O, lse, want, "fp16", L + i + 1, _v_max(V, fmt))
    for r in (0, 1, turn - 1):   # a row of the chunk is a decode step of its prefix; that call's own bar
        want = paged_decode(q[:, L + steps + r].double().cpu().numpy(), K, V, [L + steps + r + 1], table.cpu().numpy(), d ** -0.5)[0]
        err = chunk[r].double().cpu().numpy() - want[0]
        assert np.abs(err).max() <= 2e-3 and np.linalg.norm(err) <= 1e-3 * np.linalg.norm(want)
    if fmt == "fp16":
        assert torch.equal(gk, k[0]) and torch.equal(gv, v[0])


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_step_captured_in_a_graph(fmt):
    """A step of append, decode and gather, captured once: every replay takes the tokens, lengths and page ids
    of its time and gives the eager result; two graphs use one workspace in turn."""
    tm = _tm()
    dtype = torch.bfloat16
    B, Hq, Hk, d, page, per = 4, 8, 2, 128, 16, 40
    cache, ref = (tm.PagedCache.empty(B * per, page, Hk, d, FORMATS[fmt]) for _ in range(2))
    for c in (cache, ref):
        for t in (c.K, c.V, c.dK, c.dV):
            if t is not None:
                t.zero_()
    table = _table(B, per, B * per, 1100).cuda()
    start = [0, 15, 300, 555]
    lens = torch.tensor(start, dtype=torch.int32).cuda()
    total = sum(start)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(start)]), dtype=torch.int32).cuda()
    k, v = (_rows(total, Hk, d, "bf16", 1101 + i).cuda() for i in range(2))
    for c in (cache, ref):
        tm.tilemix_paged_append(c, k, v, table, lens, cu, max(start))
    newk, newv = (torch.zeros(B, 1, Hk, d, dtype=dtype, device="cuda") for _ in range(2))
    Q = torch.zeros(B, 1, Hq, d, dtype=dtype, device="cuda")
    O, lse = torch.zeros_like(Q), torch.zeros(B, Hq, device="cuda")
    gk, gv = (torch.zeros(B, 3, Hk, d, dtype=dtype, device="cuda") for _ in range(2))
    ws = torch.empty(tm.tilemix_paged_decode_workspace_size(cache, table, lens, Hq) + 256, dtype=torch.uint8, device="cuda")

    def step(c, stream=None):
        tm.tilemix_paged_append(c, newk, newv, table, lens, stream=stream)
        tm.tilemix_paged_decode(c, Q, table, lens, O=O, lse=lse, return_lse=True, workspace=ws, stream=stream)
        tm.tilemix_paged_gather(c, table, lens, 3, dtype=dtype, K=gk, V=gv, stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(cache)
        step(ref)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, torch.cuda.current_stream())
        graphs.append(g)
    torch.cuda.synchronize()
    for r in range(4):
        lens += 1
        if r == 2:
            table[1] = table[1].flip(0)          # other pages from now on
        for i, t in enumerate((newk, newv, Q)):
            t.copy_(torch.randn(t.shape, generator=_gen(1200 + 10 * r + i)).to(dtype))
        step(ref)
        torch.cuda.synchronize()
        want = [t.clone() for t in (O, lse, gk, gv)]
        for t in (O, lse, gk, gv):
            t.fill_(float("nan"))
        noise = torch.randn(1 << 20, device="cuda").sum()
        torch.cuda.synchronize()
        graphs[r % 2].replay()
        torch.cuda.synchronize()
        for a, b, name in zip((O, lse, gk, gv), want, ("O", "lse", "K", "V")):
            assert torch.equal(torch.nan_to_num(a.float(), 99.0), torch.nan_to_num(b.float(), 99.0)), (name, r)
        del noise


def test_calls_on_two_streams():
    """Concurrent calls on two streams, each with outputs and workspace of its own, and `stream` given while
    another is current."""
    tm = _tm()
    B, Hq, Hk, d, page = 3, 8, 2, 64, 32
    pool = _cached_pool("int8", (90, Hk, page, d), 1300)
    cache, table = _on_gpu(pool), _table(B, 30, 90, 1301).cuda()
    lens = torch.tensor([900, 1, 640], dtype=torch.int32).cuda()
    Qs = [torch.randn(B, 1, Hq, d, generator=_gen(1302 + i)).half().cuda() for i in range(2)]
    want = [tm.tilemix_paged_decode(cache, Q, table, lens) for Q in Qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for r in range(5):
        got += [(i, tm.tilemix_paged_decode(cache, Qs[i], table, lens, stream=streams[i])) for i in range(2)]
    torch.cuda.synchronize()
    for i, O in got:
        assert torch.equal(_bits(O), _bits(want[i]))


def test_binding_refusals():
    """Everything the binding checks, before anything is launched."""
    tm = _tm()
    cache = tm.PagedCache.empty(4, 16, 2, 64)
    table, lens = torch.zeros(3, 2, dtype=torch.int32).cuda(), torch.zeros(3, dtype=torch.int32).cuda()
    x = torch.zeros(3, 1, 2, 64, dtype=torch.float16).cuda()
    cu = torch.zeros(4, dtype=torch.int32).cuda()
    Q = torch.zeros(3, 1, 4, 64, dtype=torch.float16).cuda()
    bad = [
        lambda: tm.tilemix_paged_append(cache, x[0], x[0], table, lens),                       # packed, no cu_seqlens
        lambda: tm.tilemix_paged_append(cache, x, x, table, lens, cu, 1),                      # padded with cu_seqlens
        lambda: tm.tilemix_paged_append(cache, x[:, 0], x[:, 0], table, lens, cu),             # no max_len
        lambda: tm.tilemix_paged_append(cache, x, x[:, :, :1], table, lens),
        lambda: tm.tilemix_paged_append(cache, x, x.bfloat16(), table, lens),
        lambda: tm.tilemix_paged_append(cache, x.float(), x.float(), table, lens),
        lambda: tm.tilemix_paged_append(cache, x, x, table.long(), lens),
        lambda: tm.tilemix_paged_append(cache, x, x, table, lens[:2]),
        lambda: tm.tilemix_paged_append(cache, x, x, table[:2], lens),
        lambda: tm.tilemix_paged_append(cache, x, x, table.t().contiguous().t(), lens),        # entries not dense
        lambda: tm.tilemix_paged_append(cache, x, x, table, lens.cpu()),
        lambda: tm.tilemix_paged_append(tm.PagedCache(cache.K, cache.V), x, x, table, lens),   # no scales
        lambda: tm.tilemix_paged_append(tm.PagedCache(cache.K, cache.V[:3], cache.dK, cache.dV), x, x, table, lens),
        lambda: tm.tilemix_paged_append(tm.PagedCache(cache.K.transpose(1, 2), cache.V.transpose(1, 2), cache.dK, cache.dV),
                                        x, x, table, lens),
        lambda: tm.tilemix_paged_append(tm.PagedCache(cache.K.float(), cache.V.float()), x, x, table, lens),
        lambda: tm.tilemix_paged_append(cache, x.repeat(1, 1, 1, 2)[..., ::2], x, table, lens),
        lambda: tm.tilemix_paged_gather(cache, table, lens, 1, cu),                            # no total
        lambda: tm.tilemix_paged_gather(cache, table, lens, 0),
        lambda: tm.tilemix_paged_gather(cache, table, lens, 1, dtype=torch.float32),
        lambda: tm.tilemix_paged_gather(cache, table, lens, 1, K=x[:2], V=x),
        lambda: tm.tilemix_paged_gather(tm.PagedCache.empty(4, 16, 2, 64, torch.bfloat16), table, lens, 1, dtype=torch.float16),
        lambda: tm.tilemix_paged_decode(cache, Q[:, 0], table, lens),
        lambda: tm.tilemix_paged_decode(cache, Q[:2], table, lens),
        lambda: tm.tilemix_paged_decode(cache, Q[:, :, :3], table, lens),                      # 3 heads over 2
        lambda: tm.tilemix_paged_decode(cache, Q.float(), table, lens),
        lambda: tm.tilemix_paged_decode(cache, Q, table, lens, 0.0),
        lambda: tm.tilemix_paged_decode(cache, Q, table, lens, window=-1),
        lambda: tm.tilemix_paged_decode(cache, Q, table, lens, O=Q[:, :, :2]),
        lambda: tm.tilemix_paged_decode(cache, Q, table, lens, lse=torch.zeros(3, 3, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, ValueError, tm.TilemixError)):
            call()
            log(f"refusal {i} was accepted")
    # nothing to do is no error
    none = torch.zeros(0, 2, 64, dtype=torch.float16).cuda()
    tm.tilemix_paged_append(cache, none, none, table, lens, cu, 1)
    assert tm.tilemix_paged_gather(cache, table, lens, 1, cu, 0)[0].shape == (0, 2, 64)
