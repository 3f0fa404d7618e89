"""Host-side checks of the paged cache calls (no kernel is launched, the pointers are fake)."""

import ctypes
import os
import re

import pytest
import torch

import paper_2608_17336_amd as tm

pytestmark = pytest.mark.skipif(not os.path.exists(tm.library_path()),
                                reason="libtilemix.so not built (run __graft_entry__.build())")

OK = 0x100000
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5


class CPagedCache(ctypes.Structure):
    """tilemix_paged_cache, as the header declares it."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("format", "pages", "page_size", "heads_kv", "head_dim", "batch", "max_pages")] +
                [(n, ctypes.c_int64) for n in ("stride_k", "stride_v", "stride_dk", "stride_dv", "stride_table")] +
                [(n, ctypes.c_void_p) for n in ("K", "V", "dK", "dV", "page_table", "seqlens_k")])


def _cache(**kw):
    base = dict(format=2, pages=10, page_size=64, heads_kv=8, head_dim=128, batch=3, max_pages=5,
                stride_k=8 * 64 * 128, stride_v=8 * 64 * 128, stride_dk=512, stride_dv=512, stride_table=5,
                K=OK, V=OK, dK=OK, dV=OK, page_table=OK, seqlens_k=OK)
    base.update(kw)
    return bytes(CPagedCache(**base))


def test_packed_struct_is_the_headers():
    names = [n for n, _ in CPagedCache._fields_]
    text = open(os.path.join(os.path.dirname(tm.library_path()), "..", "include", "tilemix.h")).read()
    body = re.sub(r"/\*.*?\*/", "", text, flags=re.S).split("typedef struct tilemix_paged_cache {")[1].split("}")[0]
    assert re.findall(r"(\w+)\s*[,;]", body) == names
    values = list(range(3, 3 + len(names)))
    assert tm._PAGED.pack(*values) == bytes(CPagedCache(*values))


def _append(cache, type=0, cu=OK, length=7, total=20, K=OK, ks=1024, V=OK, vs=1024):
    return tm.load_library().tilemix_paged_append(cache, type, cu, length, total, K, ks,
                                                  V, vs, None)


def _gather(cache, type=0, cu=OK, length=7, total=20, K=OK, V=OK):
    return tm.load_library().tilemix_paged_gather(cache, type, cu, length, total, K, V,
                                                  None)


def _decode(cache, type=0, heads=32, scale=0.1, window=0, Q=OK, qs=4096, O=OK, lse=None, ws=OK, nbytes=1 << 40):
    return tm.load_library().tilemix_paged_decode(cache, type, heads, scale, window, Q,
                                                  qs, O, lse, ws, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(format=4), UNSUPPORTED), (dict(format=-1), UNSUPPORTED),
    (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED),
    (dict(page_size=48), UNSUPPORTED),
    (dict(pages=0), SHAPE), (dict(heads_kv=0), SHAPE), (dict(batch=0), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(batch=65536), SHAPE), (dict(heads_kv=65536), SHAPE),
    (dict(max_pages=(1 << 24) + 1, stride_table=1 << 25), SHAPE),
    (dict(stride_table=4), SHAPE),
    (dict(stride_k=8 * 64 * 128 - 16), SHAPE), (dict(stride_v=8 * 64 * 128 + 8), SHAPE),
    (dict(stride_dk=511), SHAPE), (dict(stride_dv=514), SHAPE),
    (dict(K=None), NULL), (dict(V=None), NULL), (dict(dK=None), NULL), (dict(dV=None), NULL),
    (dict(page_table=None), NULL), (dict(seqlens_k=None), NULL),
    (dict(K=OK + 8), ALIGN), (dict(V=OK + 1), ALIGN), (dict(dK=OK + 4), ALIGN), (dict(dV=OK + 8), ALIGN),
    (dict(page_table=OK + 2), ALIGN), (dict(seqlens_k=OK + 1), ALIGN),
])
def test_cache_refusals(kw, status):
    for call in (_append, _gather, _decode):
        assert call(_cache(**kw)) == status, call
        assert tm.load_library().tilemix_last_error()


def test_null_cache_and_types():
    for call in (_append, _gather, _decode):
        assert call(None) == NULL
        assert call(_cache(), type=2) == UNSUPPORTED
        assert call(_cache(format=1), type=0) == UNSUPPORTED     # a 16-bit pool and rows of another type
        assert call(_cache(format=0), type=1) == UNSUPPORTED
    assert tm.load_library().tilemix_paged_decode_workspace_size(None, 32, None) == NULL
    assert tm.load_library().tilemix_paged_decode_workspace_size(_cache(), 32, None) == NULL


def test_16bit_pools_need_no_scales():
    none = dict(dK=None, dV=None, stride_dk=0, stride_dv=0)
    assert _append(_cache(format=0, **none), total=0) == 0
    assert _decode(_cache(format=1, **none), type=1, Q=None) == NULL   # passed the cache's checks


def test_rows_refusals():
    for call in (_append, _gather):
        assert call(_cache(), length=0) == SHAPE
        assert call(_cache(), length=(1 << 28) + 1) == SHAPE
        assert call(_cache(), total=-1) == SHAPE
        assert call(_cache(), total=(1 << 28) + 1) == SHAPE
        assert call(_cache(), total=(1 << 24) + 1) == SHAPE            # x 8 heads x 128 channels
        assert call(_cache(), cu=None, length=7, total=20) == SHAPE    # not batch * len
        assert call(_cache(), cu=OK + 2) == ALIGN
        assert call(_cache(), K=None) == NULL
        assert call(_cache(), V=None) == NULL
        assert call(_cache(), K=OK + 8) == ALIGN
        assert call(_cache(), V=OK + 2) == ALIGN
        assert call(_cache(), total=0, K=None, V=None) == 0            # nothing to do
    assert _append(_cache(), ks=-8) == SHAPE
    assert _append(_cache(), vs=1028) == SHAPE


def test_decode_refusals():
    assert _decode(_cache(), heads=0) == SHAPE
    assert _decode(_cache(), heads=30) == SHAPE
    assert _decode(_cache(), heads=65536) == SHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _decode(_cache(), scale=scale) == SHAPE
    assert _decode(_cache(), window=-1) == SHAPE
    assert _decode(_cache(), qs=-8) == SHAPE
    assert _decode(_cache(), qs=4100) == SHAPE
    assert _decode(_cache(), Q=None) == NULL
    assert _decode(_cache(), O=None) == NULL
    assert _decode(_cache(), Q=OK + 8) == ALIGN
    assert _decode(_cache(), O=OK + 2) == ALIGN
    assert _decode(_cache(), lse=OK + 2) == ALIGN


def test_binding_refuses_host_tensors():
    pool = tm.PagedCache.empty(4, 16, 2, 64, device="cpu")
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, 1, 2, 64, dtype=torch.float16)
    for call in (lambda: tm.tilemix_paged_append(pool, x, x, table, lens),
                 lambda: tm.tilemix_paged_gather(pool, table, lens, 1),
                 lambda: tm.tilemix_paged_decode(pool, x, table, lens)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def _workspace(cache, heads=32):
    n = ctypes.c_size_t()
    assert tm.load_library().tilemix_paged_decode_workspace_size(cache, heads, ctypes.byref(n)) == 0
    return n.value


def test_decode_workspace():
    """A long page table needs one, a short one none; it is checked before anything runs."""
    long, short = _cache(max_pages=100, stride_table=100), _cache(max_pages=8, stride_table=8)
    need = _workspace(long)
    assert need > 0 and need % 256 == 0 and _workspace(short) == 0
    assert _decode(long, ws=None) == WORKSPACE
    assert _decode(long, nbytes=need - 1) == WORKSPACE
    assert _decode(long, nbytes=0) == WORKSPACE
    assert _decode(long, ws=OK + 128, nbytes=need) == ALIGN


def test_decode_of_too_large_batches():
    """What the numbering of a batch's tiles cannot hold."""
    big = dict(max_pages=1 << 24, stride_table=1 << 24)              # 2^30 tokens: 2^25 tiles of 32
    assert _workspace(_cache(batch=3, **big), heads=8) > 0
    for kw, heads in ((dict(batch=4), 8), (dict(batch=1, heads_kv=32, stride_k=32 * 64 * 128, stride_v=32 * 64 * 128,
                                                stride_dk=2048, stride_dv=2048), 32), (dict(batch=1), 8 * 16 * 4)):
        assert _decode(_cache(**big, **kw), heads=heads) == SHAPE, kw


def test_packed_rows_of_nothing():
    """A packed batch in which no sequence has a row, whose longest then has 0; but no rows and a length do not pair
    otherwise."""
    for call in (_append, _gather):
        assert call(_cache(), length=0, total=0, K=None, V=None) == 0
        assert call(_cache(), length=0, total=0, cu=None) == SHAPE
        assert call(_cache(), length=0, total=1) == SHAPE
        assert call(_cache(), length=-1, total=0) == SHAPE
        assert call(_cache(page_size=8), length=0, total=0) == UNSUPPORTED     # the cache is checked all the same
