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
