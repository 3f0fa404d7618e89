"""GPU: the MXFP4 cache on either side of where its kernels change - capacities at which sequences are split, batches
that are streamed past the caches, gathers whose results are."""

import ctypes

import numpy as np
import pytest
import torch

from gpu_util import log
from oracle.paged import paged_decode
from test_gpu_mxfp4 import TYPES, _cached_pool, _check_decode, _on_gpu, _same, _values
from test_gpu_paged import _gen

pytestmark = pytest.mark.gpu


def _tm():
    import paper_2608_17336_amd as tm
    return tm


def _workspace(cache, table, lens, heads):
    """Bytes that a decode step needs: none where no sequence is split."""
    tm = _tm()
    n = ctypes.c_size_t(0)
    tm._check(tm.load_library().tilemix_paged_decode_workspace_size(tm._paged(cache, table, lens)[0], heads, ctypes.byref(n)))
    return n.value


def _of_capacity(dtype, Hq, Hk, d, page, lens, per, whole):
    """A decode step whose page table has `per` entries a sequence, in a pool of the pages that they need."""
    tm = _tm()
    B, need = len(lens), [-(-n // page) for n in lens]
    order = torch.randperm(sum(need), generator=_gen(11)).to(torch.int32)
    table = torch.full((B, per), 2 ** 31 - 1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    pool = _cached_pool((sum(need), Hk, page, d), 12)
    cache = _on_gpu(pool)
    Q = torch.randn(B, 1, Hq, d, generator=_gen(13)).to(TYPES[dtype])
    args = (table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    assert (_workspace(cache, *args, Hq) == 0) == whole
    name = f"capacity {per * page} of {B} x {Hk} d{d} {dtype}"
    log(f"decode {name}: start")
    O, lse = tm.tilemix_paged_decode(cache, Q.cuda(), *args, return_lse=True)
    torch.cuda.synchronize()
    V = _values(pool, 1)
    _check_decode(name, O, lse, paged_decode(Q.double().numpy()[:, 0], _values(pool, 0), V, lens, table.numpy(), d ** -0.5), dtype, max(lens), V)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("beside", [-32, 0, 32])
@pytest.mark.parametrize("B,Hq,Hk,d,tiles", [(3, 4, 1, 64, 16), (3, 2, 2, 128, 16), (63, 4, 2, 64, 16), (70, 4, 2, 128, 16), (95, 2, 2, 64, 16),
                                             (64, 8, 4, 64, 32), (191, 4, 2, 128, 32), (96, 4, 4, 64, 64), (200, 2, 2, 128, 64),
                                             (256, 6, 3, 64, 64), (257, 3, 3, 128, 32), (390, 2, 2, 64, 32)])
def test_capacities_in_tiles_of_64_keys(dtype, B, Hq, Hk, d, tiles, beside):
    """Page tables of half a tile less than the most with which no sequence is split, of as many, and of half a tile
    more: for few sequences and KV heads, for 128, 192 and 384 of them and for more than there are workgroups at once."""
    slots = 64 * tiles + beside
    lens = [slots, slots - 1, 0, 1] + [(b * 41 + 5) % 90 for b in range(4, B + 4)]
    _of_capacity(dtype, Hq, Hk, d, 32, lens[:B], slots // 32, beside <= 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("Hq,Hk", [(16, 8), (64, 4)])
def test_decode_streamed_past_the_caches(dtype, d, page, Hq, Hk):
    """Codes of more than 2^27 bytes, for heads in pairs of columns and not, in pages of whole tiles and of less.  Few
    pages, each named many times (a prefix that sequences share)."""
    tm = _tm()
    pages, n = 1280 // page, 2 ** 27 // (Hk * d) + 3000
    lens = [n - 1234, 0, 1, 1500]
    assert Hq // Hk <= 16 and sum(lens) * Hk * d > 2 ** 27     # K and V, d / 2 bytes a row each
    pool = _cached_pool((pages, Hk, page, d), 21)
    table = torch.randint(0, pages, (len(lens), -(-max(lens) // page)), generator=_gen(22)).to(torch.int32)
    Q = torch.randn(len(lens), 1, Hq, d, generator=_gen(23)).to(TYPES[dtype])
    args = (_on_gpu(pool), Q.cuda(), table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda())
    log(f"decode of a large batch {dtype} d{d} page {page} {Hq}/{Hk}: start")
    O, lse = tm.tilemix_paged_decode(*args, return_lse=True)
    torch.cuda.synchronize()
    # Equal tokens count alike: the oracle's softmax over a token per (page, slot), weighted by how often it occurs.
    K, V = _values(pool, 0), _values(pool, 1)
    q, G, B = Q.double().numpy()[:, 0], Hq // Hk, len(lens)
    want = [np.zeros((B, Hq, d)), np.full((B, Hq), -np.inf), np.zeros((B, Hq, d)), np.zeros((B, Hq))]
    for b, L in enumerate(lens):
        if not L:
            continue
        t = np.arange(L)
        times = np.bincount(table[b].numpy()[t // page] * page + t % page, minlength=pages * page)
        for hq in range(Hq):
            k, v = K[:, hq // G].reshape(-1, d), V[:, hq // G].reshape(-1, d)
            s = d ** -0.5 * (k @ q[b, hq])
            m = s[times > 0].max()
            w = times * np.exp(np.minimum(s - m, 0))
            z = w.sum()
            want[0][b, hq], want[1][b, hq], want[2][b, hq] = w @ v / z, m + np.log(z), w @ np.abs(v) / z
            want[3][b, hq] = d ** -0.5 * (np.abs(k) @ np.abs(q[b, hq])).max()
    _check_decode(f"streamed {dtype} d{d} page {page} {Hq}/{Hk}", O, lse, want, dtype, max(lens), V)
    again = tm.tilemix_paged_decode(*args)
    assert torch.equal(again.view(torch.int16), O.view(torch.int16)), "the same call twice"


@pytest.mark.parametrize("fmt", ["mxfp4", "int8", "e4m3", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
def test_gather_past_the_caches_in_bf16(fmt, d):
    """More than 160 MiB of BF16 rows at once, of two sequences, are those of several calls."""
    tm = _tm()
    page, Hk, L, short = 32, 1024 // d, 41001, 777
    n = L + short
    assert 4 * n * Hk * d >= 160 << 20
    if fmt == "mxfp4":
        cache = _on_gpu(_cached_pool((16, Hk, page, d), 31))
    else:
        cache = tm.PagedCache.empty(16, page, Hk, d, {"int8": torch.int8, "e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16}[fmt])
        x = torch.randn(1, 16 * page, Hk, d, generator=_gen(32)).bfloat16().cuda()
        tm.tilemix_paged_append(cache, x, x * 2, torch.arange(16, dtype=torch.int32).view(1, 16).cuda(),
                                torch.tensor([16 * page], dtype=torch.int32).cuda())
    table = torch.randint(0, 16, (2, -(-L // page)), generator=_gen(33)).to(torch.int32)
    table[0, 5] = -1
    table, lens = table.cuda(), torch.tensor([L, short], dtype=torch.int32).cuda()
    cu = torch.tensor([0, L, n], dtype=torch.int32).cuda()
    K, V = tm.tilemix_paged_gather(cache, table, lens, L, cu, n, dtype=torch.bfloat16)
    for lo, hi in ((0, 20000), (20000, 40000), (40000, L)):
        k, v = tm.tilemix_paged_gather(cache, table[:1], lens[:1] - (L - hi), hi - lo, dtype=torch.bfloat16)
        assert _same(K[lo:hi], k[0]) and _same(V[lo:hi], v[0])
    k, v = tm.tilemix_paged_gather(cache, table[1:], lens[1:], short, dtype=torch.bfloat16)
    assert _same(K[L:], k[0]) and _same(V[L:], v[0]) and not K[5 * page:6 * page].any()
