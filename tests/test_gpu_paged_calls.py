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


@pytest.mark.parametrize("fmt", ["fp16", "int8"])
@pytest.mark.parametrize("per", [1, 80])
def test_largest_batch(fmt, per):
    """65535 sequences, most of them short or empty, in short page tables (no sequence can be split) and in long ones:
    rows written packed, read back, and attended to, against elementary operations in float64."""
    tm = _tm()
    B, Hk, Hq, d, page, pages = 65535, 1, 2, 64, 16, 65535 + 79
    g = torch.Generator().manual_seed(70)
    new = torch.randint(0, 3, (B,), generator=g)
    lens = new + torch.randint(0, 14, (B,), generator=g)
    if per > 1:
        lens[[0, 31000, B - 1]] = torch.tensor([1200, 1280, 700])
    table = torch.full((B, per), -1, dtype=torch.int32)
    table[:, 0] = torch.randperm(B, generator=g).to(torch.int32)
    for b in (0, 31000, B - 1):                                      # these share what lies behind their first pages
        table[b, 1:] = torch.arange(B, B + per - 1, dtype=torch.int32)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)])
    total = int(cu[-1])
    new_gpu, t_gpu, l_gpu, cu_gpu = new.cuda(), table.cuda(), lens.to(torch.int32).cuda(), cu.to(torch.int32).cuda()
    shape = (pages, Hk, page, d)
    pool = [torch.randn(shape, generator=g).half() if fmt == "fp16" else torch.randint(-127, 128, shape, generator=g).to(torch.int8) for _ in "KV"]
    scales = [torch.rand(shape[:3], generator=g) / 64 for _ in "KV"] if fmt == "int8" else [None, None]
    cache = tm.PagedCache(*[None if t is None else t.cuda() for t in pool + scales])
    rows = [torch.randn(total, Hk, d, generator=g).half().cuda() for _ in "KV"]
    tm.tilemix_paged_append(cache, *rows, t_gpu, l_gpu, cu_gpu, 2)
    got = tm.tilemix_paged_gather(cache, t_gpu, l_gpu, 2, cu_gpu, total)
    torch.cuda.synchronize()
    for x, y in zip(rows, got):
        x, y = x.double(), y.double()
        half = 0.0 if fmt == "fp16" else x.abs().amax(-1, keepdim=True) / 254
        assert ((x - y).abs() <= half * (1 + 2.0 ** -10) + y.abs() * 2.0 ** -11 * (fmt == "int8")).all()
    # Every row is where its sequence has it: the last tokens of the sequences.
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), new_gpu)
    t = l_gpu.long()[b] - new_gpu[b] + torch.arange(total, device="cuda") - cu.cuda()[b]
    id_, slot = t_gpu.long()[b, t // page], t % page
    for X, S, y in zip(cache[:2], cache[2:], got):
        held = X[id_, :, slot].float()
        assert torch.equal((held if S is None else held * S[id_, :, slot][..., None]).half(), y)

    Q = torch.randn(B, 1, Hq, d, generator=g).half().cuda()
    O, lse = tm.tilemix_paged_decode(cache, Q, t_gpu, l_gpu, return_lse=True)
    torch.cuda.synchronize()
    values = [X.double() if S is None else X.double() * S.double()[..., None] for X, S in zip(cache[:2], cache[2:])]
    eps = torch.finfo(torch.float16).eps

    def check(k, v, seen, bs):
        """k, v [n, tokens, d], seen [n, tokens]: sequences bs."""
        q = Q[bs, 0].double()
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * d ** -0.5
        s = s.masked_fill(~seen[:, None], float("-inf"))
        want_lse = torch.logsumexp(s, -1)
        p = torch.exp(s - want_lse.clamp(min=-1e300)[..., None])
        want, mass = torch.matmul(p, v), torch.matmul(p, v.abs())
        n = seen.shape[1]
        ds = (d + 8) * 2.0 ** -24 * 0.125 * torch.matmul(q.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1)
        tol = eps / 2 * want.abs() + 2.0 ** -25 + (2 * ds[..., None] + 2.0 ** -20 + n * 2.0 ** -23) * mass + n * 2.0 ** -39 * v.abs().amax()
        assert ((O[bs, 0].double() - want).abs() <= tol * (1 + eps)).all()
        some = torch.isfinite(want_lse)
        assert torch.equal(torch.isfinite(lse[bs]), some) and not O[bs, 0][~some].any()
        assert ((lse[bs].double() - want_lse)[some].abs() <= (ds + n * 2.0 ** -24 + 2.0 ** -20)[some]).all()

    first = t_gpu[:, 0].long()
    short = torch.arange(B, device="cuda")[l_gpu <= page]
    check(*[x[first[short], 0] for x in values], torch.arange(page, device="cuda") < l_gpu[short, None], short)
    for b in (0, 31000, B - 1) if per > 1 else ():
        ids = t_gpu[b].long()
        check(*[x[ids, 0].reshape(1, -1, d) for x in values], (torch.arange(per * page, device="cuda") < int(lens[b]))[None],
              torch.tensor([b], device="cuda"))
