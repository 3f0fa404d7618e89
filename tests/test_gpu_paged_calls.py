"""GPU: calls of the paged cache's binding at the edges of their arguments."""

import pytest
import torch

from test_gpu_paged import FORMATS, _tm

pytestmark = pytest.mark.gpu


def _small(fmt="fp16"):
    """A pool of 4 pages for 3 sequences, their page table and lengths (0), rows and offsets of none."""
    tm = _tm()
    cache = tm.PagedCache.empty(4, 16, 2, 64, FORMATS[fmt])
    table, lens = torch.zeros(3, 2, dtype=torch.int32).cuda(), torch.zeros(3, dtype=torch.int32).cuda()
    return cache, table, lens, torch.zeros(0, 2, 64, dtype=torch.float16).cuda(), torch.zeros(4, dtype=torch.int32).cuda()


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
def test_packed_rows_of_nothing(fmt):
    """A packed batch that brings no row; its longest sequence has 0."""
    tm = _tm()
    cache, table, lens, none, cu = _small(fmt)
    tm.tilemix_paged_append(cache, none, none, table, lens, cu, 0)
    K, V = tm.tilemix_paged_gather(cache, table, lens, 0, cu, 0)
    assert K.shape == V.shape == (0, 2, 64)


@pytest.mark.parametrize("beyond", [2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 40 + 7, -2 ** 32 + 1])
def test_numbers_past_32_bits(beyond):
    """No length, window or number of heads is taken modulo 2^32."""
    tm = _tm()
    cache, table, lens, _, cu = _small()
    x = torch.zeros(5, 2, 64, dtype=torch.float16).cuda()
    Q = torch.zeros(3, 1, 2, 64, dtype=torch.float16).cuda()
    out = [torch.zeros(5, 2, 64, dtype=torch.float16, device="cuda") for _ in "KV"]
    for call in (lambda: tm.tilemix_paged_append(cache, x, x, table, lens, cu, beyond),
                 lambda: tm.tilemix_paged_gather(cache, table, lens, beyond, cu, K=out[0], V=out[1]),
                 lambda: tm.tilemix_paged_gather(cache, table, lens, 1, cu, beyond),
                 lambda: tm.tilemix_paged_gather(cache, table, lens, beyond),
                 lambda: tm.tilemix_paged_decode(cache, Q, table, lens, window=beyond),
                 lambda: tm.tilemix_paged_decode_workspace_size(cache, table, lens, beyond)):
        with pytest.raises((ValueError, tm.TilemixError)):
            call()
    torch.cuda.synchronize()


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
def test_broken_offsets_touch_no_other_rows(fmt):
    """cu_seqlens that step back or point outside the rows, every row of another value: append takes the rows that the
    clamped offsets name and none behind `total` (NaN there), gather writes those and none behind (9 there)."""
    tm = _tm()
    Hk, d, page, total, guard = 2, 64, 16, 20, 40
    cache = tm.PagedCache.empty(8, page, Hk, d, FORMATS[fmt])
    for t in cache:
        if t is not None:
            t.zero_()
    table = torch.arange(8, dtype=torch.int32).view(4, 2).cuda()
    lens = torch.tensor([30, 30, 30, 30], dtype=torch.int32).cuda()
    cu = torch.tensor([-5, 12, 3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32).cuda()
    bufs = []
    for sign in (1.0, -1.0):   # constant rows: any format holds their values to half a step of FP16
        x = torch.full((total + guard, Hk, d), float("nan"), dtype=torch.float16)
        x[:total] = sign * torch.arange(1, total + 1).view(-1, 1, 1)
        bufs.append(x.cuda())
    tm.tilemix_paged_append(cache, bufs[0][:total], bufs[1][:total], table, lens, cu, 2 ** 20)
    torch.cuda.synchronize()
    owned = {0: (0, 12), 1: (12, 0), 2: (3, 17), 3: (20, 0)}         # first row and number of rows, clamped
    for X, S, buf in ((cache.K, cache.dK, bufs[0]), (cache.V, cache.dV, bufs[1])):
        held = X.float() if S is None else X.float() * S[..., None]
        held = held.half().transpose(1, 2).reshape(4, 2 * page, Hk, d).cpu()
        for b, (first, n) in owned.items():
            assert torch.equal(held[b, 30 - n:30], buf[first:first + n].cpu())
            assert not held[b, :30 - n].any() and not held[b, 30:].any()
    outs = [torch.full((total + guard, Hk, d), 9.0, dtype=torch.float16, device="cuda") for _ in "KV"]
    tm.tilemix_paged_gather(cache, table, lens, 2 ** 20, cu, K=outs[0][:total], V=outs[1][:total])
    torch.cuda.synchronize()
    for out, buf in zip(outs, bufs):
        out, buf = out.cpu(), buf.cpu()
        assert (out[total:] == 9.0).all()
        assert torch.equal(out[:3], buf[:3]) and torch.equal(out[12:total], buf[12:total])
        for r in range(3, 12):   # of sequence 0 or of sequence 2, where row r is what append read there
            assert ((out[r] == buf[r]).all(-1)).all()
