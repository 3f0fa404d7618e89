"""GPU: the paged key/value cache in MXFP4 - append and gather bit for bit, decode against float64."""

import numpy as np
import pytest
import torch

from gpu_util import log
from oracle.paged import block_codes, mx_values, new_tokens, pack_e2m1, paged_decode, slot_of
import test_gpu_paged
from test_gpu_paged import _bits, _gen, _rows, _table, _words

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
E2M1, E8M0 = torch.float4_e2m1fn_x2, torch.float8_e8m0fnu


def _tm():
    import paper_2608_17336_amd as tm
    return tm


def _random_pool(shape, seed):
    """Bytes (CPU) K, V [P, H, page, d / 2], dK, dV [P, H, page, d / 32] of arbitrary bits."""
    g = _gen(seed)
    P, H, page, d = shape
    return [torch.randint(0, 256, (P, H, page, d // n), generator=g, dtype=torch.uint8) for n in (2, 2, 32, 32)]


def _on_gpu(pool):
    K, V, dK, dV = (t.cuda() for t in pool)
    return _tm().PagedCache(K.view(E2M1), V.view(E2M1), dK.view(E8M0), dV.view(E8M0))


def _host(cache):
    return [t.view(torch.uint8).cpu() for t in cache]


def _write(pool, x, op, page, slot):
    """Oracle: row x [Hk, d] of operand op (0 K, 1 V) into (page, slot) of a CPU pool."""
    codes, byte = block_codes(x.double().numpy())
    pool[op][page, :, slot] = torch.from_numpy(pack_e2m1(codes))
    pool[op + 2][page, :, slot] = torch.from_numpy(byte)


def _same_pool(cache, pool):
    for name, a, b in zip(("K", "V", "dK", "dV"), _host(cache), pool):
        bad = a != b
        assert not bad.any(), f"{name}: {int(bad.sum())} bytes differ, first at {bad.nonzero()[0].tolist()}"


def _values(pool, op):
    return mx_values(pool[op].numpy(), pool[op + 2].numpy())


def _read(pool, op, page, slot, dtype):
    """Oracle: the values of a row, rounded once."""
    v = mx_values(pool[op][page, :, slot].numpy(), pool[op + 2][page, :, slot].numpy())
    return torch.from_numpy(v).to(TYPES[dtype])


def _same(a, b):
    """Bit for bit; a NaN has any payload."""
    nan = torch.isnan(a) & torch.isnan(b)
    return bool(((_bits(a) == _bits(b)) | nan.cpu()).all())


# ------------------------------------------------------------------------- append and gather

@pytest.mark.parametrize("d,page,Hk", [(64, 16, 1), (64, 256, 3), (128, 64, 8), (128, 32, 2), (128, 16, 33)])
@pytest.mark.parametrize("dtype", TYPES)
def test_append_then_gather_packed(dtype, d, page, Hk):
    """Ragged packed rows, written and read back bit for bit; nothing else changes."""
    tm = _tm()
    new = [0, 1, 2 * page + 3, page, 17]
    old = [5, 0, page - 2, 0, 3 * page + 1]
    B, per, pages = len(new), 6, 40
    lens = [o + n for o, n in zip(old, new)]
    cu = np.concatenate([[0], np.cumsum(new)])
    total = int(cu[-1]) + 4                                          # four rows that no sequence owns
    pool = _random_pool((pages, Hk, page, d), d + page)
    table = _table(B, per, pages, 1)
    K, V = _rows(total, Hk, d, dtype, 2), _rows(total, Hk, d, dtype, 3)
    cache = _on_gpu(pool)
    t_gpu, l_gpu = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    cu_gpu = torch.tensor(cu, dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), t_gpu, l_gpu, cu_gpu, max(new))
    rows = [(r, *slot_of(table.numpy(), pages, page, b, t)) for b, r, t in new_tokens(lens, cu, B, max(new), total)]
    for r, p, s in rows:
        _write(pool, K[r], 0, p, s)
        _write(pool, V[r], 1, p, s)
    torch.cuda.synchronize()
    _same_pool(cache, pool)

    outK, outV = (torch.full((total, Hk, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in "KV")
    tm.tilemix_paged_gather(cache, t_gpu, l_gpu, max(new), cu_gpu, K=outK, V=outV)
    for x, op, out in ((K, 0, outK), (V, 1, outV)):
        want = torch.full((total, Hk, d), 7.0, dtype=TYPES[dtype])
        for r, p, s in rows:
            want[r] = _read(pool, op, p, s, dtype)
        assert _same(out.cpu(), want), "KV"[op]
        # At most half a step of its block, a quarter or half of 2^e below 2 and 4, 2^e beyond; 2^e <= 2 a / 7.
        x, got = x.double()[: int(cu[-1])], out.cpu().double()[: int(cu[-1])]
        unit = x.unflatten(-1, (-1, 32)).abs().amax(-1, keepdim=True) * 2 / 7
        f = torch.finfo(TYPES[dtype])
        assert ((got - x).unflatten(-1, (-1, 32)).abs() <= unit + got.unflatten(-1, (-1, 32)).abs() * f.eps / 2 + f.tiny).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,L,Hk,d", [(1, 1, 1, 64), (70, 1, 2, 128), (3, 5, 8, 128), (2, 130, 2, 64)])
def test_append_padded_and_strided(dtype, B, L, Hk, d):
    """[B, L, Hk, d] rows that are slices of a fused projection; pages that are slices of a tensor of K and
    V; a page table that is a slice; sequences that are shorter than L."""
    tm = _tm()
    page, per = 16, 10
    pages = B * per + 1
    K0, V0, dK0, dV0 = _random_pool((pages, Hk, page, d), 5)
    both, scales = torch.stack([K0, V0], 1), torch.stack([dK0, dV0], 1)
    lens = [int(x) for x in torch.randint(0, per * page, (B,), generator=_gen(7))]
    lens[0] = min(L, 3)
    wide = torch.full((B, per + 2), -7, dtype=torch.int32)
    wide[:, :per] = _table(B, per, pages, 8)
    table = wide[:, :per]
    fused = _rows(B * L, 3 * Hk, d, dtype, 9).view(B, L, 3 * Hk, d)
    K, V = fused[:, :, Hk:2 * Hk], fused[:, :, 2 * Hk:]
    gb, gs, gf = both.cuda(), scales.cuda(), fused.cuda()
    cache = tm.PagedCache(gb[:, 0].view(E2M1), gb[:, 1].view(E2M1), gs[:, 0].view(E8M0), gs[:, 1].view(E8M0))
    l_gpu, t_gpu = torch.tensor(lens, dtype=torch.int32).cuda(), wide.cuda()[:, :per]
    tm.tilemix_paged_append(cache, gf[:, :, Hk:2 * Hk], gf[:, :, 2 * Hk:], t_gpu, l_gpu)
    pool = [both[:, 0], both[:, 1], scales[:, 0], scales[:, 1]]
    for b, r, t in new_tokens(lens, None, B, L, B * L):
        at = slot_of(table.numpy(), pages, page, b, t)
        if at:
            _write(pool, K[b, r - b * L], 0, *at)
            _write(pool, V[b, r - b * L], 1, *at)
    torch.cuda.synchronize()
    _same_pool(cache, pool)
    gK, gV = tm.tilemix_paged_gather(cache, t_gpu, l_gpu, L, dtype=TYPES[dtype])
    assert gK.shape == gV.shape == (B, L, Hk, d)
    short = L - lens[0]                                              # rows before the first token are zeros
    assert not gK[0, :short].any() and not gV[0, :short].any()


@pytest.mark.parametrize("dtype", TYPES)
def test_append_rows_without_a_slot(dtype):
    """Missing pages, tokens past the page table, lengths below the new rows: nothing is written there, and
    reading gives zeros."""
    tm = _tm()
    page, per, pages, Hk, d = 16, 3, 12, 2, 128
    table = _table(4, per, pages, 11)
    table[0, 1], table[1, 0], table[2, 2] = -1, pages, 2 ** 31 - 1
    lens, new = [40, 20, 55, -5], [30, 20, 50, 6]
    cu = np.concatenate([[0], np.cumsum(new)])
    total = int(cu[-1])
    pool = _random_pool((pages, Hk, page, d), 12)
    cache = _on_gpu(pool)
    K, V = _rows(total, Hk, d, dtype, 13), _rows(total, Hk, d, dtype, 14)
    args = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    cu_gpu = torch.tensor(cu, dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), *args, cu_gpu, 50)
    missing = []
    for b, r, t in new_tokens(lens, cu, 4, 50, total):
        at = slot_of(table.numpy(), pages, page, b, t)
        if at:
            _write(pool, K[r], 0, *at)
            _write(pool, V[r], 1, *at)
        else:
            missing.append(r)
    torch.cuda.synchronize()
    _same_pool(cache, pool)
    assert len(missing) > 30
    gK, gV = tm.tilemix_paged_gather(cache, *args, 50, cu_gpu, total, dtype=TYPES[dtype])
    assert not gK[missing].any() and not gV[missing].any()
    kept = [r for r in range(total) if r not in missing]
    assert gK[kept].any(-1).any(-1).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_append_every_value(dtype, d):
    """Every number of the type, and every pair of neighbours in it, in blocks whose exponent another value sets:
    rounding, ties, subnormal numbers, infinities, NaN and zeros of both signs."""
    tm = _tm()
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    x = bits.view(TYPES[dtype])
    order = torch.argsort(x.abs().float().nan_to_num(nan=float("inf")), stable=True)
    sorted_rows = x[order].view(-1, 1, d)                            # blocks of neighbours: the top of a block sets 2^e
    shuffled = x[torch.randperm(65536, generator=_gen(15))]
    shuffled = torch.where(shuffled.abs() <= 8, shuffled, shuffled.sign() * 0.125).view(-1, 1, d)
    tops = shuffled.clone()                                          # one value of each block at 3.5 .. 6.99
    tops[:, 0, ::32] = torch.linspace(3.5, 6.99, tops[:, 0, ::32].numel()).view(tops[:, 0, ::32].shape).to(TYPES[dtype])
    rows = torch.cat([sorted_rows, shuffled, tops])
    n, page = rows.shape[0], 256
    pages = -(-n // page)
    pool = _random_pool((pages, 1, page, d), 16)
    cache = _on_gpu(pool)
    table, lens = torch.arange(pages, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([n], dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, rows[None].cuda(), rows.flip(0)[None].contiguous().cuda(), table, lens)
    for op, y in ((0, rows), (1, rows.flip(0))):
        codes, byte = block_codes(y[:, 0].double().numpy())
        for t0 in range(0, n, page):
            m = min(page, n - t0)
            pool[op][t0 // page, 0, :m] = torch.from_numpy(pack_e2m1(codes[t0:t0 + m]))
            pool[op + 2][t0 // page, 0, :m] = torch.from_numpy(byte[t0:t0 + m])
    torch.cuda.synchronize()
    _same_pool(cache, pool)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_gather_every_code_and_exponent(dtype, d):
    """All codes under all exponents: rounded once to the type, infinite past its range, NaN for byte 255."""
    tm = _tm()
    page, pages = 16, 16
    pool = _random_pool((pages, 1, page, d), 17)
    for e in range(256):
        p, s = e // page, e % page
        for op in (0, 1):
            codes = torch.arange(d // 2, dtype=torch.int32) + 37 * op
            both = (codes % 16) | ((codes * 3 + e) % 16) << 4
            pool[op][p, 0, s] = both.to(torch.uint8)
            pool[op + 2][p, 0, s] = e
    cache = _on_gpu(pool)
    table, lens = torch.arange(pages, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([256], dtype=torch.int32).cuda()
    got = tm.tilemix_paged_gather(cache, table, lens, 256, dtype=TYPES[dtype])
    for op in (0, 1):
        want = torch.from_numpy(_values(pool, op)).view(256, 1, d).to(TYPES[dtype])
        assert _same(got[op][0].cpu(), want), "KV"[op]


# ------------------------------------------------------------------------------------ decode

def _check_decode(name, O, lse, want, dtype, n, V):
    """As for a BF16 cache, and what FP32 and BF16 cannot hold: codes of 0 are common, so an output may be made of
    weights near FP32's smallest normal number alone.  A weight (at most 1) below 2^-126, its second piece below
    it, and a product with a value below it may count as 0: each adds at most 2^-126 max(|v|, 1) for each of n tokens,
    3 n 2^-126 (v_max + 1) in all.  That check takes n 2^-39 of what it calls v_max."""
    v_max = float(np.abs(V).max())
    test_gpu_paged._check_decode(name, O, lse, want, dtype, n, 3 * 2.0 ** (39 - 126) * (v_max + 1))


def _cached_pool(shape, seed, gain=1.0):
    """A pool (CPU) of finite rows; blocks differ in size by up to 2^6."""
    out = [None] * 4
    for op in (0, 1):
        x = torch.randn(shape, generator=_gen(seed + op)) * gain
        x = x * torch.exp2(torch.randint(-3, 4, (*shape[:3], shape[3] // 32, 1), generator=_gen(seed + 7 + op))).expand(
            -1, -1, -1, -1, 32).reshape(shape)
        codes, byte = _fast_codes(x.half())
        out[op], out[op + 2] = codes, byte
    return out


def _fast_codes(x):
    """block_codes and pack_e2m1 for finite rows of ordinary size (the oracle's own search is a loop over blocks)."""
    b = x.double().numpy().reshape(*x.shape[:-1], -1, 32)
    f, k = np.frexp(np.abs(b).max(-1))
    e = k - 3 + (f >= 0.875)
    from oracle.paged import round_e2m1
    codes = np.copysign(round_e2m1(b * np.exp2(-e.astype(np.float64))[..., None]), b).reshape(x.shape)
    return torch.from_numpy(pack_e2m1(codes)), torch.from_numpy((e + 127).astype(np.uint8))


def test_fast_codes_are_the_oracles():
    x = torch.randn(5, 64, generator=_gen(3)).half()
    codes, byte = block_codes(x.double().numpy())
    fast = _fast_codes(x)
    assert np.array_equal(fast[0].numpy(), pack_e2m1(codes)) and np.array_equal(fast[1].numpy(), byte)


def _decode_case(dtype, Hq, Hk, d, page, lens, window=0, seed=0, holes=(), gain=1.0, q_gain=1.0, per=None):
    tm = _tm()
    B = len(lens)
    per = per or max(1, max(-(-x // page) for x in lens))
    pages = B * per + 2
    table = _table(B, per, pages, seed + 30)
    for b, e, x in holes:
        table[b, e] = x
    pool = _cached_pool((pages, Hk, page, d), seed + 31, gain)
    used = torch.zeros(pages, page, dtype=torch.bool)
    for b, L in enumerate(lens):
        for t in range(max(0, L - window) if window else 0, L):
            at = slot_of(table.numpy(), pages, page, b, t)
            if at:
                used[at] = True
    for op in (0, 1):                                               # slots that do not count: NaN and the largest values
        pool[op].masked_fill_(~used[:, None, :, None], 0x7f)
        pool[op + 2].masked_fill_(~used[:, None, :, None], 255)
        pool[op + 2][::2].masked_fill_(~used[::2, None, :, None], 254)
    for b, L in enumerate(lens):                                    # page ids past a length mean nothing
        table[b, -(-max(L, 0) // page):] = 2 ** 31 - 1 if b % 2 else -1
    Q = (torch.randn(B, 1, Hq, d, generator=_gen(seed + 40)) * q_gain).to(TYPES[dtype])
    cache = _on_gpu(pool)
    args = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    name = f"mxfp4/{dtype} {Hq}/{Hk} d{d} page {page} lens {lens[:6]} window {window}"
    log(f"decode {name}: start")
    O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), *args, window=window, return_lse=True)
    torch.cuda.synchronize()
    K, V = (np.where(used.numpy()[:, None, :, None], _values(pool, op), 0.0) for op in (0, 1))
    want = paged_decode(Q.double().numpy()[:, 0], K, V, lens, table.numpy(), d ** -0.5, window)
    _check_decode(name, O, lse, want, dtype, max(lens), V)
    again = tm.tilemix_paged_decode(cache, Q.cuda(), *args, window=window)
    torch.cuda.synchronize()
    assert torch.equal(_bits(again), _bits(O)), "the same call twice"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,d,page", [(2, 2, 64, 16), (8, 1, 128, 64), (6, 2, 64, 32), (7, 1, 128, 16),
                                          (16, 1, 128, 256), (33, 3, 64, 128)])
def test_decode_lengths(dtype, Hq, Hk, d, page):
    """Lengths from none to several tiles: either side of slabs, tiles and pages."""
    _decode_case(dtype, Hq, Hk, d, page, [0, 1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 130, 255, 257, 300])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,d", [(17, 1, 128), (32, 1, 64), (40, 2, 128), (100, 1, 64)])
def test_decode_large_groups(dtype, Hq, Hk, d):
    """More query heads per KV head than one block of 16."""
    _decode_case(dtype, Hq, Hk, d, 32, [500, 3, 0, 77], seed=100)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,Hq,Hk,d,page", [([5000], 8, 2, 128, 16), ([9001, 1], 4, 1, 64, 256), ([4096, 17, 2500], 8, 2, 64, 64)])
def test_decode_long(dtype, lens, Hq, Hk, d, page):
    """Caches that are split over workgroups."""
    _decode_case(dtype, Hq, Hk, d, page, lens, seed=200)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,d,long", [(2, 2, 64, 700), (6, 1, 128, 700), (128, 1, 64, 1100), (96, 2, 128, 1100)])
def test_decode_many_sequences(dtype, Hq, Hk, d, long):
    """More sequences than lanes of a wave, with empty ones at both ends; few and many beside the workgroups that
    run at once, so that a long sequence is cut, and a workgroup has parts of several."""
    lens = [(0, 3, 37, 150, 1, 64)[b * b % 6] for b in range(150)]
    lens[7] = lens[130] = long
    lens[149] = 0
    _decode_case(dtype, Hq, Hk, d, 16, lens, seed=1500)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,d,page,long", [(6, 2, 128, 64, 1500), (128, 16, 64, 64, 1500), (96, 2, 128, 128, 1100), (40, 2, 64, 256, 2600)])
def test_decode_many_sequences_in_large_pages(dtype, Hq, Hk, d, page, long):
    """The same where a page holds whole tiles, with up to 8 query heads for a KV head and more."""
    lens = [(0, 3, 37, 150, 1, 64, 65, 200)[b * b % 8] for b in range(150)]
    lens[7] = lens[130] = long
    lens[149] = 0
    _decode_case(dtype, Hq, Hk, d, page, lens, seed=1550)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk", [(8, 1), (9, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_of_slices(dtype, Hq, Hk, d):
    """Pages of K and V that are slices of one tensor, and strided queries."""
    tm = _tm()
    for page in (16, 64):
        pool = _cached_pool((12, Hk, page, d), 1560)
        want = tm.tilemix_paged_decode(_on_gpu(pool), *(_args := (torch.randn(3, 1, Hq, d, generator=_gen(1561)).to(TYPES[dtype]).cuda(),
                                       _table(3, 4, 12, 1562).cuda(), torch.tensor([4 * page, 17, 2 * page + 5], dtype=torch.int32).cuda())))
        K, V, dK, dV = (t.cuda() for t in pool)
        both, scales = torch.stack([K, V, K], 1), torch.stack([dK, dV], 1)
        cache = tm.PagedCache(both[:, 0].view(E2M1), both[:, 1].view(E2M1), scales[:, 0].view(E8M0), scales[:, 1].view(E8M0))
        fused = torch.cat([_args[0], _args[0]], 2)
        got = tm.tilemix_paged_decode(cache, fused[:, :, Hq:], *_args[1:])
        assert torch.equal(_bits(got), _bits(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G", [8, 9])
def test_decode_keys_of_many_magnitudes(dtype, G):
    """Keys around 2^30, 1 and 2^-30 side by side in a tile, and tiles of small ones only: scores are off by FP32's share
    of the largest, and a sequence of small keys keeps their bits."""
    for exps in ((30, 0, -30), (-30, -30, -30), (-60, -30, 30)):
        tm = _tm()
        d, page, L = 128, 64, 300
        K = torch.randn(1, L, 1, d, generator=_gen(61)) * torch.exp2(torch.tensor(exps, dtype=torch.float32)[torch.arange(L) % 3])[None, :, None, None]
        V = torch.randn(1, L, 1, d, generator=_gen(62))
        Q = torch.randn(1, 1, G, d, generator=_gen(63)).to(TYPES[dtype])
        cache = tm.PagedCache(*(t.view(torch.uint8).zero_().view(t.dtype) for t in tm.PagedCache.empty(5, page, 1, d, E2M1)))
        table, lens = torch.arange(5, dtype=torch.int32).view(1, 5).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
        tm.tilemix_paged_append(cache, K.bfloat16().cuda(), V.bfloat16().cuda(), table, lens)
        scale = 2.0 ** -max(exps) / d ** 0.5
        O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, scale, return_lse=True)
        pool = _host(cache)
        want = paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), _values(pool, 1), [L], table.cpu().numpy(), scale)
        _check_decode(f"magnitudes {exps} {dtype} G{G}", O, lse, want, dtype, L, V.numpy())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,d,page", [(8, 128, 64), (9, 128, 64), (16, 128, 16), (16, 64, 64), (12, 64, 32)])
@pytest.mark.parametrize("byte,code", [(252, 6.0), (253, 3.0), (254, 1.5)])
@pytest.mark.parametrize("scale", [1.0, 8.0, 4096.0])
def test_decode_largest_keys(dtype, G, d, page, byte, code, scale):
    """Keys of 1.5 2^127, of either sign, and queries that are 0 or have one small channel: finite scores.  Those of a head are
    equal but for their sign, so that its weights are equal, or 0: off by their pieces' 2^-15, and a sum of n terms by n 2^-24.
    (Scores are FP32 in units of ln 2: with the largest scale 2^(h - 25) 1.5 2^127 4096 / ln 2 = 2.16 2^(h + 114) of heads from 13
    on is none.)"""
    tm = _tm()
    L, pages = 90, 90 // page + 1
    pool = _cached_pool((pages, 1, page, d), 1800)
    sign = torch.randint(0, 2, (pages, 1, page, d), generator=_gen(1801)).numpy() * 2.0 - 1
    pool[0] = torch.from_numpy(pack_e2m1(code * sign))
    pool[2] = torch.full((pages, 1, page, d // 32), byte, dtype=torch.uint8)
    Q = torch.zeros(1, 1, G, d)
    for h in range(1, G):
        Q[0, 0, h, (11 * h) % d] = 2.0 ** (h - 25)
    Q = Q.to(TYPES[dtype])
    table, lens = torch.arange(pages, dtype=torch.int32).view(1, -1), torch.tensor([L], dtype=torch.int32)
    O, lse = tm.tilemix_paged_decode(_on_gpu(pool), Q.cuda(), table.cuda(), lens.cuda(), scale, return_lse=True)
    V = _values(pool, 1)
    wO, wl, mass, reach = paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), V, [L], table.numpy(), scale)
    room = reach / np.log(2.0) < 2.0 ** 128
    assert room.sum() == (min(G, 13) if scale == 4096.0 else G)
    wO, wl, mass = wO[room], wl[room], mass[room]
    O, lse, f = O.double().cpu().numpy()[:, 0][room], lse.double().cpu().numpy()[room], torch.finfo(TYPES[dtype])
    assert np.isfinite(O).all() and (np.abs(O - wO) <= f.eps / 2 * np.abs(wO) + (2.0 ** -15 + L * 2.0 ** -24) * mass * (1 + f.eps) + f.smallest_normal * f.eps).all()
    assert (np.abs(lse - wl) <= 2.0 ** -21 * np.abs(wl)).all()      # four roundings, log2 e's and ln 2's among them


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("G,d,page", [(8, 128, 64), (9, 128, 64), (16, 128, 16), (16, 64, 64)])
def test_decode_small_keys_beside_a_large_one(dtype, G, d, page):
    """A tile with one key 2^32 times as large as the others, in channels that the query does not read: the others keep
    their bits."""
    tm = _tm()
    L, pages = 64, 64 // page
    K = torch.randn(1, L, 1, d, generator=_gen(1810)) * 2.0 ** -12
    K[..., :32] = 0.0
    K[0, 5, 0, :32] = 2.0 ** 20
    V = torch.randn(1, L, 1, d, generator=_gen(1811))
    Q = torch.randn(1, 1, G, d, generator=_gen(1812))
    Q[..., :32] = 0.0
    Q = Q.to(TYPES[dtype])
    cache = tm.PagedCache.empty(pages, page, 1, d, E2M1)
    table, lens = torch.arange(pages, dtype=torch.int32).view(1, -1).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K.bfloat16().cuda(), V.bfloat16().cuda(), table, lens)
    scale = 2.0 ** 12 / d ** 0.5
    O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, scale, return_lse=True)
    pool = _host(cache)
    want = paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), _values(pool, 1), [L], table.cpu().numpy(), scale)
    _check_decode(f"beside a large key {dtype} G{G} d{d}", O, lse, want, dtype, L, _values(pool, 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,B,slots", [(4, 3, 480), (4, 3, 512), (4, 3, 544), (64, 64, 992), (64, 64, 1024), (64, 64, 1056),
                                        (128, 140, 256)])
def test_decode_capacities(dtype, Hq, B, slots):
    """Page tables of 15 to 17 and 31 to 33 tiles of 32 keys, full and empty sequences, one or several a workgroup."""
    lens = [slots, slots - 1, 0, 1] + [(b * 41 + 5) % 170 for b in range(4, B)]
    _decode_case(dtype, Hq, 1, 64, 32, lens[:B], seed=1600, per=slots // 32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("window", [1, 16, 50, 64, 1000])
def test_decode_window(dtype, window):
    """The last tokens only; the pages before them are given back (-1)."""
    lens, page = [0, 1, 49, 50, 51, 64, 200, 1313], 16
    holes = [(b, e, -1) for b, L in enumerate(lens) for e in range(max(0, L - window) // page)]
    _decode_case(dtype, 8, 2, 128, page, lens, window=window, seed=300, holes=holes)
    _decode_case(dtype, 6, 3, 64, 128, lens, window=window, seed=301)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 256])
def test_decode_missing_pages(dtype, page):
    """Tokens without a page are left out; a sequence without any page gets 0."""
    lens = [3 * page, 5 * page - 3, 2 * page]
    holes = [(0, 1, -1), (1, 0, 2 ** 30), (1, 3, -2 ** 31), (2, 0, -1), (2, 1, 10 ** 6)]
    _decode_case(dtype, 8, 2, 128, page, lens, seed=400, holes=holes)


@pytest.mark.parametrize("dtype", TYPES)
def test_decode_sharp_scores(dtype):
    """Scores of some hundreds (one token takes all the weight) and of nearly nothing (all alike)."""
    _decode_case(dtype, 8, 2, 128, 64, [700, 129], seed=500, q_gain=60.0)
    _decode_case(dtype, 8, 2, 128, 64, [700, 129], seed=501, q_gain=2.0 ** -10)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens", [[262000, 0, 1, 100], [90000, 93000, 81100]])
def test_decode_of_a_large_batch(dtype, lens):
    """Caches larger than 2^27 bytes.  Few pages, each named many times (a prefix that sequences share)."""
    tm = _tm()
    d, page, pages, Hk, Hq = 128, 64, 20, 8, 16
    assert sum(lens) * 2 * Hk * d // 2 > 2 ** 27
    pool = _cached_pool((pages, Hk, page, d), 1700)
    table = torch.randint(0, pages, (len(lens), -(-max(lens) // page)), generator=_gen(1701)).to(torch.int32)
    Q = torch.randn(len(lens), 1, Hq, d, generator=_gen(1702)).to(TYPES[dtype])
    log(f"decode of a large batch {dtype} {lens}: start")
    O, lse = tm.tilemix_paged_decode(_on_gpu(pool), Q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), return_lse=True)
    torch.cuda.synchronize()
    # Equal tokens count alike: the oracle's softmax over a token per (page, slot), weighted by how often it occurs.
    K, V = _values(pool, 0), _values(pool, 1)
    times = np.zeros((len(lens), pages, page))
    for b, L in enumerate(lens):
        t = np.arange(L)
        np.add.at(times[b], (table[b].numpy()[t // page], t % page), 1)
    q = Q.double().numpy()[:, 0]
    want = [np.zeros((len(lens), Hq, d)), np.full((len(lens), Hq), -np.inf), np.zeros((len(lens), Hq, d)), np.zeros((len(lens), Hq))]
    for b, hq in np.ndindex(len(lens), Hq):
        if not lens[b]:
            continue
        k, v = K[:, hq // 2].reshape(-1, d), V[:, hq // 2].reshape(-1, d)
        s = d ** -0.5 * (k @ q[b, hq])
        m = s[times[b].ravel() > 0].max()
        w = times[b].ravel() * np.exp(np.minimum(s - m, 0))
        z = w.sum()
        want[0][b, hq], want[1][b, hq], want[2][b, hq] = w @ v / z, m + np.log(z), w @ np.abs(v) / z
        want[3][b, hq] = d ** -0.5 * (np.abs(k) @ np.abs(q[b, hq])).max()
    _check_decode(f"large batch {dtype}", O, lse, want, dtype, max(lens), V)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_decode_query_magnitudes(dtype, d):
    """Query channels from the type's smallest numbers to large ones side by side, in every order of blocks, and
    keys that single one channel out: no channel's bits are lost beside a larger one's."""
    tm = _tm()
    page, L = 64, d
    small = 2.0 ** -24 if dtype == "fp16" else 2.0 ** -100
    steps = torch.logspace(np.log10(small), np.log10(200.0), d, dtype=torch.float64)
    mant = 1 + torch.rand(d, generator=_gen(41), dtype=torch.float64)
    Q = torch.stack([steps * mant, steps.flip(0) * mant, (steps * mant)[torch.randperm(d, generator=_gen(42))],
                     steps[torch.randperm(d, generator=_gen(43))] * torch.where(mant > 1.5, 1.0, -1.0)]).to(TYPES[dtype]).view(1, 1, 4, d)
    K = torch.zeros(L, 1, d)
    K[torch.arange(L), 0, torch.arange(L)] = 1.5                     # token t reads channel t
    V = torch.randn(L, 1, d, generator=_gen(44))
    cache = tm.PagedCache.empty(2, page, 1, d, E2M1)
    table, lens = torch.arange(2, dtype=torch.int32).view(1, 2).cuda(), torch.tensor([L], dtype=torch.int32).cuda()
    tm.tilemix_paged_append(cache, K[None].to(TYPES[dtype]).cuda(), V[None].to(TYPES[dtype]).cuda(), table, lens)
    pool = _host(cache)
    for t in range(0, L, 7):                                         # one token at a time: its score alone
        one = torch.full((1, 2), -1, dtype=torch.int32)
        p = t // page
        one[0, 0] = p
        O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), one.cuda(), torch.tensor([t % page + 1], dtype=torch.int32).cuda(),
                                         1.0, window=1, return_lse=True)
        s = Q.double()[0, 0, :, t] * 1.5                             # exact in FP32 but for its own rounding and log2 e
        assert ((lse[0].double().cpu() - s).abs() <= s.abs() * 2.0 ** -21 + 2.0 ** -126).all(), t
    O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, return_lse=True)
    want = paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), _values(pool, 1), [L], table.cpu().numpy(), d ** -0.5)
    _check_decode(f"query magnitudes {dtype}", O, lse, want, dtype, L, V.numpy())


@pytest.mark.parametrize("gains", [(2.0 ** 60, 2.0 ** -60, 2.0 ** -60), (2.0 ** -60, 2.0 ** 60, 2.0 ** 60),
                                   (2.0 ** 115, 2.0 ** 110, 2.0 ** -110), (2.0 ** -110, 2.0 ** -110, 2.0 ** 115)])
def test_decode_bf16_range(gains):
    """Rows and queries over BF16's range."""
    tm = _tm()
    gk, gv, gq = gains
    for d in (64, 128):
        page, L = 16, 90
        K = (torch.randn(1, L, 1, d, generator=_gen(700)) * gk).bfloat16()
        V = (torch.randn(1, L, 1, d, generator=_gen(701)) * gv).bfloat16()
        V[:, ::3] *= 2.0 ** -10
        Q = (torch.randn(1, 1, 3, d, generator=_gen(702)) * gq).bfloat16()
        cache = tm.PagedCache.empty(6, page, 1, d, E2M1)
        table = torch.arange(6, dtype=torch.int32).view(1, 6).cuda()
        lens = torch.tensor([L], dtype=torch.int32).cuda()
        tm.tilemix_paged_append(cache, K.cuda(), V.cuda(), table, lens)
        O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), table, lens, return_lse=True)
        torch.cuda.synchronize()
        pool = _host(cache)
        want = paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), _values(pool, 1), [L], table.cpu().numpy(), d ** -0.5)
        _check_decode(f"range {gk:g} d{d}", O, lse, want, "bf16", L, V.double().numpy())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [2, 10])
def test_decode_nan_stays_in_its_sequence(dtype, d, G):
    """A NaN block in one sequence's keys reaches that sequence's heads and nobody else; one in its values those
    channels of its heads."""
    tm = _tm()
    page = 16
    pool = _cached_pool((12, 2, page, d), 800)
    table = _table(3, 4, 12, 801)
    lens = torch.tensor([60, 60, 60], dtype=torch.int32).cuda()
    Q = torch.randn(3, 1, 2 * G, d, generator=_gen(802)).to(TYPES[dtype]).cuda()
    before = tm.tilemix_paged_decode(_on_gpu(pool), Q, table.cuda(), lens)
    at = (int(table[1, 2]), 1, 5)                                    # token 37 of sequence 1, KV head 1
    for op in (0, 1):
        bad = [t.clone() for t in pool]
        bad[op][at] = 0
        bad[op + 2][at][1] = 255
        after = tm.tilemix_paged_decode(_on_gpu(bad), Q, table.cuda(), lens)
        hit = torch.zeros_like(before, dtype=torch.bool)
        hit[1, 0, G:, slice(None) if op == 0 else slice(32, 64)] = True
        assert torch.isnan(after[hit]).all() and not torch.isnan(after[~hit]).any()
        if op == 0:
            assert torch.equal(_bits(after[~hit]), _bits(before[~hit]))


def test_offsets_past_32_bits():
    """A pool whose pages lie beyond 2^32 bytes, read and written at its end."""
    tm = _tm()
    page, Hk, d = 256, 8, 128
    each = page * Hk * d // 2
    pages = 2 ** 32 // each + 20
    K, V = (torch.empty((pages, Hk, page, d // 2), dtype=torch.uint8, device="cuda").view(E2M1) for _ in "KV")
    cache = tm.PagedCache(K, V, *(torch.empty((pages, Hk, page, d // 32), dtype=torch.uint8, device="cuda").view(E8M0) for _ in "KV"))
    table = torch.tensor([[pages - 1, 0, pages - 7], [1, pages - 2, pages - 3]], dtype=torch.int32).cuda()
    lens = torch.tensor([600, 513], dtype=torch.int32).cuda()
    cu = torch.tensor([0, 600, 1113], dtype=torch.int32).cuda()
    x, y = (_rows(1113, Hk, d, "bf16", 950 + i).cuda() for i in range(2))
    x, y = x.clamp(-4, 4), y.clamp(-4, 4)
    small = tm.PagedCache.empty(6, page, Hk, d, E2M1)
    st = torch.arange(6, dtype=torch.int32).view(2, 3).cuda()
    Q = torch.randn(2, 1, 16, d, generator=_gen(960)).bfloat16().cuda()
    got = []
    for c, t in ((cache, table), (small, st)):
        tm.tilemix_paged_append(c, x, y, t, lens, cu, 600)
        got.append((*tm.tilemix_paged_gather(c, t, lens, 600, cu, 1113, dtype=torch.bfloat16), tm.tilemix_paged_decode(c, Q, t, lens)))
    for a, b in zip(*got):
        assert torch.equal(_bits(a), _bits(b))


@pytest.mark.parametrize("fmt", ["mxfp4", "int8", "fp16"])
@pytest.mark.parametrize("d,Hk", [(64, 3), (128, 8)])
def test_append_of_many_tiles(fmt, d, Hk):
    """A packed batch of thousands of tokens fills the pool as its sequences do one by one in pieces, and nothing else; the
    rows behind the last sequence are read by nobody and written by nobody."""
    tm = _tm()
    page, new = 16, [1, 4999, 0, 333, 2048, 7, 1201]
    old = [5, 0, 9, 15, 100, 16, 3]
    B, n, behind = len(new), sum(new), 41
    per = max(-(-(o + x) // page) for o, x in zip(old, new))
    P = B * per
    table = _table(B, per, P, 1920).cuda()
    lens = torch.tensor([o + x for o, x in zip(old, new)], dtype=torch.int32).cuda()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
    k, v = (torch.randn(n + behind, Hk, d, generator=_gen(1921 + i)).half().cuda() for i in range(2))
    dtype = {"mxfp4": E2M1, "int8": torch.int8, "fp16": torch.float16}[fmt]
    bits = lambda c: [t.view(torch.uint8) for t in c if t is not None]
    one, ref = (tm.PagedCache.empty(P, page, Hk, d, dtype) for _ in range(2))
    for c in (one, ref):
        for t in bits(c):
            t.fill_(77)
    tm.tilemix_paged_append(one, k, v, table, lens, cu, max(new))
    for b in range(B):
        for lo in range(0, new[b], 64):
            m = min(64, new[b] - lo)
            at = slice(int(cu[b]) + lo, int(cu[b]) + lo + m)
            tm.tilemix_paged_append(ref, k[None, at], v[None, at], table[b:b + 1], torch.tensor([old[b] + lo + m], dtype=torch.int32).cuda())
    for x, y in zip(bits(one), bits(ref)):
        assert torch.equal(x, y)
    gk, gv = (torch.full((n + behind, Hk, d), 3.0, dtype=torch.float16, device="cuda") for _ in range(2))
    tm.tilemix_paged_gather(one, table, lens, max(new), cu, n + behind, K=gk, V=gv, dtype=torch.float16)
    assert (gk[n:] == 3).all() and (gv[n:] == 3).all()
    for b in range(B):
        if new[b]:
            for lo in range(0, new[b], 64):
                m = min(64, new[b] - lo)
                x, y = tm.tilemix_paged_gather(one, table[b:b + 1], torch.tensor([old[b] + lo + m], dtype=torch.int32).cuda(), m)
                at = slice(int(cu[b]) + lo, int(cu[b]) + lo + m)
                assert _same(gk[at], x[0]) and _same(gv[at], y[0])


@pytest.mark.parametrize("fmt", ["mxfp4", "int8", "bf16"])
def test_gather_of_many_rows(fmt):
    """More than 2^27 bytes of rows at once are those of several calls."""
    tm = _tm()
    Hk, d, page, L = 8, 128, 64, 33000
    P = -(-L // page)
    if fmt == "mxfp4":
        cache = _on_gpu(_cached_pool((16, Hk, page, d), 1900))
    else:
        cache = tm.PagedCache.empty(16, page, Hk, d, {"int8": torch.int8, "bf16": torch.bfloat16}[fmt])
        x = torch.randn(1, 16 * page, Hk, d, generator=_gen(1901)).bfloat16().cuda()
        tm.tilemix_paged_append(cache, x, x * 2, torch.arange(16, dtype=torch.int32).view(1, 16).cuda(),
                                torch.tensor([16 * page], dtype=torch.int32).cuda())
    table = torch.randint(0, 16, (1, P), generator=_gen(1902)).to(torch.int32)
    table[0, 5] = -1
    lens = torch.tensor([L], dtype=torch.int32).cuda()
    assert 4 * L * Hk * d > 2 ** 27
    K, V = tm.tilemix_paged_gather(cache, table.cuda(), lens, L, dtype=torch.bfloat16)
    for lo in range(0, L, 11000):
        k, v = tm.tilemix_paged_gather(cache, table.cuda(), lens - (L - lo - 11000), 11000, dtype=torch.bfloat16)
        assert _same(K[:, lo:lo + 11000], k) and _same(V[:, lo:lo + 11000], v)
    assert not K[0, 5 * page:6 * page].any()


@pytest.mark.parametrize("fmt", ["mxfp4", "int8", "e4m3", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_gather_past_the_caches(fmt, d):
    """More than 2^28 bytes of rows at once, of two sequences in pages that lie in any order, are those of several calls."""
    tm = _tm()
    page, Hk, L, short = 32, 1024 // d, 67001, 777
    P, n = -(-L // page), 67001 + 777
    if fmt == "mxfp4":
        cache = _on_gpu(_cached_pool((16, Hk, page, d), 1910))
    else:
        dtype = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn, "fp16": torch.float16}[fmt]
        cache = tm.PagedCache.empty(16, page, Hk, d, dtype)
        x = torch.randn(1, 16 * page, Hk, d, generator=_gen(1911)).half().cuda()
        tm.tilemix_paged_append(cache, x, x * 2, torch.arange(16, dtype=torch.int32).view(1, 16).cuda(),
                                torch.tensor([16 * page], dtype=torch.int32).cuda())
    table = torch.randint(0, 16, (2, P), generator=_gen(1912)).to(torch.int32).cuda()
    lens = torch.tensor([L, short], dtype=torch.int32).cuda()
    cu = torch.tensor([0, L, n], dtype=torch.int32).cuda()
    assert 4 * n * Hk * d > 2 ** 28
    K, V = tm.tilemix_paged_gather(cache, table, lens, L, cu, n, dtype=torch.float16)
    for lo, hi in ((0, 20000), (20000, 40000), (40000, L)):
        k, v = tm.tilemix_paged_gather(cache, table[:1], lens[:1] - (L - hi), hi - lo, dtype=torch.float16)
        assert _same(K[lo:hi], k[0]) and _same(V[lo:hi], v[0])
    k, v = tm.tilemix_paged_gather(cache, table[1:], lens[1:], short, dtype=torch.float16)
    assert _same(K[L:], k[0]) and _same(V[L:], v[0])


# ------------------------------------------------------------------------------- as they are used

def test_prefill_append_decode_and_chunked_prefill():
    """A prompt through tilemix_prefill and into the cache, steps of append and decode, then the next
    turn's rows against the prefix that is read back, through tilemix_prefill_varlen."""
    tm = _tm()
    Hq, Hk, d, page, L, steps, turn = 8, 2, 128, 64, 333, 5, 70
    g = _gen(1000)
    n = L + steps + turn
    q, k, v = (torch.randn(1, n, H, d, generator=g).half().cuda() for H in (Hq, Hk, Hk))
    cache = tm.PagedCache(*(t.view(torch.uint8).zero_().view(t.dtype) for t in tm.PagedCache.empty(12, page, Hk, d, E2M1)))
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
    pool = _host(cache)
    K, V = (np.nan_to_num(_values(pool, op)) for op in (0, 1))
    for i, (O, lse) in enumerate(outs):
        want = paged_decode(q[:, L + i].double().cpu().numpy(), K, V, [L + i + 1], table.cpu().numpy(), d ** -0.5)
        _check_decode(f"step {i} mxfp4", O, lse, want, "fp16", L + i + 1, V)
    for r in (0, 1, turn - 1):   # a row of the chunk is a decode step of its prefix; that call's own bar
        want = paged_decode(q[:, L + steps + r].double().cpu().numpy(), K, V, [L + steps + r + 1], table.cpu().numpy(), d ** -0.5)[0]
        err = chunk[r].double().cpu().numpy() - want[0]
        assert np.abs(err).max() <= 2e-3 and np.linalg.norm(err) <= 1e-3 * np.linalg.norm(want)


def test_calls_on_two_streams():
    """Concurrent decodes and gathers on two streams, each with results and workspace of its own, and `stream` given while
    another is current."""
    tm = _tm()
    B, Hq, Hk, d, page = 3, 8, 2, 128, 64
    cache, table = _on_gpu(_cached_pool((90, Hk, page, d), 1300)), _table(B, 30, 90, 1301).cuda()
    lens = torch.tensor([1900, 1, 1640], dtype=torch.int32).cuda()
    Qs = [torch.randn(B, 1, Hq, d, generator=_gen(1302 + i)).half().cuda() for i in range(2)]
    want = [tm.tilemix_paged_decode(cache, Q, table, lens) for Q in Qs]
    rows = tm.tilemix_paged_gather(cache, table, lens, 700)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for r in range(5):
        got += [(i, tm.tilemix_paged_decode(cache, Qs[i], table, lens, stream=streams[i]),
                 tm.tilemix_paged_gather(cache, table, lens, 700, stream=streams[1 - i])) for i in range(2)]
    torch.cuda.synchronize()
    for i, O, kv in got:
        assert torch.equal(_bits(O), _bits(want[i]))
        assert all(_same(x, y) for x, y in zip(kv, rows))


def test_step_captured_in_a_graph():
    """A step of append, decode and gather, captured in two graphs that share a workspace: every replay takes the
    tokens and lengths of its time and gives the eager result."""
    tm = _tm()
    dtype = torch.bfloat16
    B, Hq, Hk, d, page, per = 4, 8, 2, 128, 16, 40
    cache, ref = (tm.PagedCache(*(t.view(torch.uint8).zero_().view(t.dtype) for t in tm.PagedCache.empty(B * per, page, Hk, d, E2M1)))
                  for _ in range(2))
    table = _table(B, per, B * per, 1100).cuda()
    start = [0, 15, 300, 555]
    lens = torch.tensor(start, dtype=torch.int32).cuda()
    cu = torch.tensor(np.concatenate([[0], np.cumsum(start)]), dtype=torch.int32).cuda()
    k, v = (_rows(sum(start), Hk, d, "bf16", 1101 + i).cuda() for i in range(2))
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

    step(cache)
    step(ref)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(cache, torch.cuda.current_stream())
        graphs.append(graph)
    torch.cuda.synchronize()
    for r in range(4):
        lens += 1
        for i, t in enumerate((newk, newv, Q)):
            t.copy_(torch.randn(t.shape, generator=_gen(1200 + 10 * r + i)).to(dtype))
        for t in (O, lse, gk, gv):
            t.fill_(float("nan"))
        graphs[r % 2].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (O, lse, gk, gv)]
        step(ref)
        torch.cuda.synchronize()
        for a, b in zip(got, (O, lse, gk, gv)):
            assert torch.equal(_bits(a), _bits(b)), r
        for a, b in zip(_host(cache), _host(ref)):
            assert torch.equal(a, b), r
