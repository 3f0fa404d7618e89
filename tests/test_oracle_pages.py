"""Pins of oracle/pages.py, and the host-side refusals of tilemix_paged_reserve and tilemix_rotary."""

import ctypes
import os
import random

import pytest
import torch

import paper_2608_17336_amd as tm
from oracle.pages import reserve

built = pytest.mark.skipif(not os.path.exists(tm.library_path()), reason="libtilemix.so not built (run __graft_entry__.build())")


def test_by_hand():
    """Three sequences: one grows into a second page, one is done, one begins; the ring wraps."""
    got = reserve([[7, -1], [3, 4], [-1, -1]], [15, 20, 0], [18, 0, 5], 16, [8, 9, 5, 6, 0], 2, 3, total=10)
    assert got["table"] == [[7, 5], [-1, -1], [6, -1]]
    assert (got["head"], got["count"], got["refused"]) == (4, 3, 0)         # 0, and 3 and 4 behind it
    assert got["ids"] == [3, 4, 5, 6, 0]
    assert got["seqlens"] == [18, 0, 5] and got["cu_seqlens"] == [0, 3, 3, 8]
    assert got["positions"] == [15, 16, 17, 0, 1, 2, 3, 4, -1, -1]
    assert got["slots"] == [7 * 16 + 15, 80, 81, 96, 97, 98, 99, 100, -1, -1]


def test_refusals_by_hand():
    """The second asks for more than there is; the third, behind it, is refused too; the fourth needs none."""
    got = reserve([[-1] * 3] * 3 + [[9, -1, -1]], [0, 0, 0, 3], [16, 48, 1, 9], 16, [1, 2, 3], 0, 3, total=4)
    assert got["seqlens"] == [16, 0, 0, 9] and got["refused"] == 2 and got["cu_seqlens"] == [0, 16, 16, 16, 22]
    assert got["table"][0][0] == 1 and got["count"] == 2
    assert reserve([[-1]], [0], [17], 16, [1, 2], 0, 2)["refused"] == 1      # past the page table


def test_window_by_hand():
    got = reserve([[4, 5, 6, -1, -1, -1]], [40], [90], 16, [9, 8, 7, 1], 0, 4, window=20, total=50)
    # Of 90 tokens the last 20 are seen: entries 4 and 5.  0 .. 2 go back, 3 gets no page.
    assert got["table"] == [[-1, -1, -1, -1, 9, 8]] and got["count"] == 2 and got["first"] == [4]
    assert got["ids"] == [9, 8, 7, 1]                                        # no room for 4, 5, 6 in a list of four: lost
    assert got["slots"][:24] == [-1] * 24 and got["slots"][24:] == [9 * 16 + i for i in range(16)] + [8 * 16 + i for i in range(10)]


def test_no_page_is_lost_or_doubled():
    """Random steps: every page is free or in one place of one table."""
    rng = random.Random(3)
    for window in (0, 50):
        B, per, page, P = 6, 9, 16, 30
        table, lens = [[-1] * per for _ in range(B)], [0] * B
        ids, head, count, first = list(range(P)), 0, P, [0] * B
        for _ in range(200):
            want = [rng.choice([0, n, n + 1, n + 1, n + 1, n + rng.randrange(80), max(0, n - 20)]) for n in lens]
            got = reserve(table, lens, want, page, ids, head, count, window, first)
            table, lens, ids, head, count, first = (got[k] for k in ("table", "seqlens", "ids", "head", "count", "first"))
            free = [ids[(head + i) % P] for i in range(count)]
            used = [p for b, row in enumerate(table) for p in row[first[b]:-(-lens[b] // page)]]
            assert sorted(free + used) == list(range(P))


# ------------------------------------------------------------------------------------ refusals

OK = 0x100000
NULL, SHAPE, UNSUPPORTED, ALIGN = 1, 2, 3, 4


def _reserve(**kw):
    a = dict(page_size=16, batch=3, max_pages=5, table=OK, stride=5, lens=OK, wanted=OK, window=0, first=None, ids=OK, capacity=10, state=OK,
             state_out=OK, lens_out=OK, cu=None, positions=None, slots=None, total=0)
    a.update(kw)
    return tm.load_library().tilemix_paged_reserve(*a.values(), None)


@built
@pytest.mark.parametrize("kw,status", [
    (dict(page_size=8), UNSUPPORTED), (dict(page_size=24), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(page_size=0), UNSUPPORTED),
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=(1 << 26) + 1, stride=1 << 27), SHAPE),
    (dict(stride=4), SHAPE), (dict(stride=1 << 41), SHAPE), (dict(window=-1), SHAPE), (dict(capacity=0), SHAPE),
    (dict(capacity=(1 << 30) - 1), SHAPE), (dict(total=-1), SHAPE), (dict(total=(1 << 28) + 1), SHAPE),
    *[({k: None}, NULL) for k in ("table", "lens", "wanted", "ids", "state", "state_out", "lens_out")],
    *[({k: OK + 2}, ALIGN) for k in ("table", "lens", "wanted", "ids", "state", "state_out", "lens_out", "cu", "positions")],
    (dict(slots=OK + 4), ALIGN), (dict(window=5), NULL), (dict(window=5, first=OK + 1), ALIGN),
])
def test_reserve_refusals(kw, status):
    assert _reserve(**kw) == status
    assert tm.load_library().tilemix_last_error()


def _rotary(positions=OK, lens=None, cu=None, batch=1, total=6, Q=OK, qs=512, Qo=OK + 4096, qos=512, K=OK, ks=256, Ko=OK + 4096, kos=256, **kw):
    p = dict(type=0, layout=0, d=128, r=64, Hq=4, Hk=2, inverse=0, magnitude=1.0, freq=OK)
    p.update(kw)
    c = tm._ROTARY.pack(*p.values()) if p["freq"] is not None else tm._ROTARY.pack(*[*p.values()][:-1], 0)
    return tm.load_library().tilemix_rotary(c, positions, lens, cu, batch, total, Q, qs, Qo, qos, K, ks, Ko, kos, None)


@built
@pytest.mark.parametrize("kw,status", [
    (dict(type=2), UNSUPPORTED), (dict(type=5), UNSUPPORTED), (dict(layout=2), UNSUPPORTED), (dict(layout=-1), UNSUPPORTED),
    (dict(d=96), UNSUPPORTED), (dict(r=0), SHAPE), (dict(r=63), SHAPE), (dict(r=130), SHAPE), (dict(d=64, r=66), SHAPE),
    (dict(Hq=0, Hk=0), SHAPE), (dict(Hq=-1), SHAPE), (dict(Hk=65536), SHAPE), (dict(magnitude=float("nan")), SHAPE),
    (dict(total=-1), SHAPE), (dict(total=(1 << 28) + 1), SHAPE), (dict(positions=None, lens=OK, batch=0), SHAPE),
    (dict(positions=None, lens=OK, batch=65536), SHAPE), (dict(positions=None, lens=OK, batch=4), SHAPE), (dict(positions=None), NULL),
    (dict(qs=-8), SHAPE), (dict(ks=252), SHAPE), (dict(qos=504), SHAPE), (dict(kos=248), SHAPE), (dict(qos=1 << 41), SHAPE),
    (dict(Q=None), NULL), (dict(Ko=None), NULL), (dict(freq=None), NULL), (dict(freq=OK + 4), ALIGN),
    (dict(Q=OK + 8), ALIGN), (dict(Qo=OK + 2), ALIGN), (dict(K=OK + 4), ALIGN), (dict(positions=OK + 1), ALIGN),
    (dict(positions=None, lens=OK + 2), ALIGN), (dict(positions=None, lens=OK, cu=OK + 2), ALIGN),
    (dict(Qo=OK, qs=1024), SHAPE),                                            # in place, with another stride
])
def test_rotary_refusals(kw, status):
    assert _rotary(**kw) == status
    assert tm.load_library().tilemix_last_error()


@built
def test_rotary_of_nothing():
    assert _rotary(total=0, Q=None, K=None, Qo=None, Ko=None, freq=None) == 0
    assert tm.load_library().tilemix_rotary(None, OK, None, None, 1, 1, OK, 0, OK, 0, None, 0, None, 0, None) == NULL


@built
def test_binding_refuses_host_tensors():
    i32 = torch.int32
    z = torch.zeros(2, dtype=i32)
    with pytest.raises(TypeError, match="CUDA"):
        tm.tilemix_paged_reserve(tm.PageList.full(4, "cpu"), torch.zeros(2, 2, dtype=i32), z, z, 16)
    x = torch.zeros(2, 2, 64, dtype=torch.float16)
    with pytest.raises(TypeError, match="CUDA"):
        tm.tilemix_rotary(x, None, torch.ones(8, dtype=torch.float64), z)
    lst = tm.PageList.full(5, "cpu")
    assert lst.ids.tolist() == [0, 1, 2, 3, 4] and lst.state.tolist() == [0, 5, 0, 0]
