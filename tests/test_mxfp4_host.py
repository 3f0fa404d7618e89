"""Host-side checks of the paged cache calls over an MXFP4 pool (no kernel is launched, the pointers are fake)."""

import os
import subprocess

import pytest
import torch

import paper_2608_17336_amd as tm
from test_paged_host import ALIGN, NULL, OK, SHAPE, UNSUPPORTED, _append, _cache, _decode, _gather, _workspace

pytestmark = pytest.mark.skipif(not os.path.exists(tm.library_path()),
                                reason="libtilemix.so not built (run __graft_entry__.build())")


def _mx(**kw):
    return _cache(**{**dict(format=5, stride_k=8 * 64 * 64, stride_v=8 * 64 * 64, stride_dk=8 * 64 * 4, stride_dv=8 * 64 * 4), **kw})


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(format=6), UNSUPPORTED),
    (dict(stride_k=8 * 64 * 64 - 16), SHAPE), (dict(stride_v=8 * 64 * 64 + 8), SHAPE), (dict(stride_k=1 << 41), SHAPE),
    (dict(stride_dk=8 * 64 * 4 - 16), SHAPE), (dict(stride_dv=8 * 64 * 4 + 4), SHAPE), (dict(stride_dk=-16), SHAPE),
    (dict(dK=None), NULL), (dict(dV=None), NULL), (dict(K=None), NULL),
    (dict(K=OK + 8), ALIGN), (dict(dK=OK + 4), ALIGN), (dict(dV=OK + 1), ALIGN),
])
def test_cache_refusals(kw, status):
    for call in (_append, _gather, _decode):
        assert call(_mx(**kw)) == status, call
        assert tm.load_library().tilemix_last_error()


def test_both_types_are_taken():
    for type in (0, 1):
        assert _append(_mx(), type=type, total=0) == 0
        assert _decode(_mx(), type=type, Q=None) == NULL               # passed the cache's checks
    for type in (2, 3, 5):
        assert _append(_mx(), type=type) == UNSUPPORTED
    assert _workspace(_mx(max_pages=100, stride_table=100)) > 0


def test_smallest_strides_are_a_pages():
    """Pages may follow one another without a gap; d = 64: 32 bytes of codes and 2 exponents a row."""
    small = dict(head_dim=64, heads_kv=1, page_size=16, stride_k=16 * 32, stride_v=16 * 32, stride_dk=32, stride_dv=32)
    assert _append(_mx(**small), total=0) == 0
    assert _append(_mx(**{**small, "stride_dv": 16}), total=0) == SHAPE


def test_binding_refusals():
    pool = tm.PagedCache.empty(4, 16, 2, 64, torch.float4_e2m1fn_x2, device="cpu")
    assert pool.K.shape == (4, 2, 16, 32) and pool.dV.shape == (4, 2, 16, 2) and pool.dV.dtype == torch.float8_e8m0fnu
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(1, 1, 2, 64, dtype=torch.float16)
    for call in (lambda: tm.tilemix_paged_append(pool, x, x, table, lens),
                 lambda: tm.tilemix_paged_gather(pool, table, lens, 1),
                 lambda: tm.tilemix_paged_decode(pool, x, table, lens)):
        with pytest.raises(TypeError, match="CUDA"):
            call()


def test_a_torch_without_the_4_bit_type(monkeypatch):
    """Everything but MXFP4 pools works with a torch that has no such type."""
    monkeypatch.delattr(torch, "float4_e2m1fn_x2")
    monkeypatch.delattr(torch, "float8_e8m0fnu")
    monkeypatch.setattr(tm, "_TORCH", None)
    monkeypatch.setattr(tm, "_FORMATS", {})
    pool = tm.PagedCache.empty(4, 16, 2, 64, device="cpu")
    assert pool.K.dtype == torch.int8 and pool.dK.dtype == torch.float32
    assert tm.PagedCache.empty(4, 16, 2, 64, torch.bfloat16, device="cpu").dK is None
    assert [tm._format(t) for t in (torch.float16, torch.bfloat16, torch.int8, torch.float8_e4m3fn, torch.float64)] == [0, 1, 2, 3, -1]
    assert tm._alloc(None, (3,), dtype=torch.int32).shape == (3,)


@pytest.mark.parametrize("compiler,name", [("gcc", "use.c"), ("g++", "use.cpp")])
def test_scales_keep_their_type_in_c(tmp_path, compiler, name):
    """FP32 scales are written and read back as such, by name and by position; exponents are bytes behind the same pointers."""
    src = tmp_path / name
    src.write_text('''
#include "tilemix.h"
float first(const tilemix_paged_cache* c) { const float* s = c->dK; float* v = c->dV; return s[0] + v[0]; }
void bytes(tilemix_paged_cache* c, uint8_t* e) { c->dK = (float*)e; c->dV = (float*)(e + 16); }
tilemix_paged_cache make(void* x, float* s, const int32_t* t) {
  tilemix_paged_cache c = {TILEMIX_INT8, 4, 16, 2, 64, 1, 4, 2048, 2048, 32, 32, 4, x, x, s, s + 32, t, t};
  float* back = c.dK;
  c.dV = back;
  return c;
}
''')
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    r = subprocess.run([compiler, "-fsyntax-only", "-Wall", "-Werror", "-I", include, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
