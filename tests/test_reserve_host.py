"""Host-side checks of tilemix_paged_reserve (no kernel is launched, the pointers are fake)."""

import os

import pytest

import paper_2608_17336_amd as tm

pytestmark = pytest.mark.skipif(not os.path.exists(tm.library_path()),
                                reason="libtilemix.so not built (run __graft_entry__.build())")

NULL, SHAPE = 1, 2
STEP = 1 << 40                                 # addresses further apart than any of them is long
NAMES = ("table", "lens", "wanted", "first", "ids", "state", "state_out", "lens_out", "cu", "positions", "slots")
BYTES = dict(lens=4 * 2000, wanted=4 * 2000, first=4 * 2000, ids=4 * 50, state=16, state_out=16, lens_out=4 * 2000, cu=4 * 2001,
             positions=4 * 300, slots=8 * 300)


def _reserve(window=0, B=2000, per=8, stride=10, page=16, total=300, capacity=50, **at):
    p = {name: (1 + i) * STEP for i, name in enumerate(NAMES)}
    p.update(at)
    return tm.load_library().tilemix_paged_reserve(page, B, per, p["table"], stride, p["lens"], p["wanted"], window, p["first"], p["ids"],
                                                   capacity, p["state"], p["state_out"], p["lens_out"], p["cu"], p["positions"], p["slots"],
                                                   total, None)


WRITTEN = [n for n in NAMES if n not in ("lens", "wanted", "table")]


@pytest.mark.parametrize("other", [n for n in NAMES if n != "table"])
@pytest.mark.parametrize("name", WRITTEN)
def test_overlaps_are_refused(name, other):
    """What is written, over the first, a middle or the last word of anything else; also over all of it, but for the new
    lengths and the new state over the old."""
    if name == other:
        return
    at = (1 + NAMES.index(other)) * STEP
    same = (name, other) in (("lens_out", "lens"), ("lens_out", "wanted"), ("state_out", "state"), ("state", "state_out"))
    for shift in [BYTES[other] - 8, 8, 8 - BYTES[name]] + ([] if same else [0]):
        shift = shift // 8 * 8                 # (slots are 8-byte aligned)
        assert _reserve(window=5, **{name: at + shift}) == SHAPE, shift
        assert b"overlap" in tm.load_library().tilemix_last_error()


@pytest.mark.parametrize("name", [n for n in NAMES if n != "table"])
def test_overlaps_with_the_table_are_refused(name):
    """Rows of 8 entries, 10 apart: over the first and last row, out of the gap into a row, from the row before it."""
    table, row, last = STEP, 40, 40 * 1999
    for at in (table, table + 24, table + last, table + last + 24, table + 32 + 7 * row, table - BYTES[name] + 8):
        if name in ("state", "state_out") and at == table - BYTES[name] + 8:
            at = table - 8
        assert _reserve(window=5, **{name: at}) == SHAPE, at - table
        assert b"overlap" in tm.load_library().tilemix_last_error()


def test_overlaps_through_a_shifted_alias():
    """The new lengths are the old ones, but the wanted ones are those a place further on; prefix sums over the lengths they are
    made of."""
    lens = 2 * STEP
    assert _reserve(lens_out=lens, wanted=lens + 4) == SHAPE
    assert _reserve(cu=lens - 4) == SHAPE and _reserve(cu=3 * STEP - 4) == SHAPE
    assert _reserve(lens_out=lens, wanted=lens, first=lens, window=3) == SHAPE
    assert _reserve(state_out=6 * STEP, state=6 * STEP, cu=6 * STEP + 8) == SHAPE


def test_entries_that_the_window_leaves_are_counted_in_32_bits():
    """With a window a call may set every entry of the table: up to 2^30 - 1 of them.  (NULL: passed the checks of sizes.)"""
    many = dict(B=64, per=1 << 24, stride=1 << 24, page=64)
    assert _reserve(window=1, **many) == SHAPE and b"window" in tm.load_library().tilemix_last_error()
    assert _reserve(window=1, **{**many, "B": 65, "per": (1 << 24) - 1}) == SHAPE
    assert _reserve(window=1, table=None, **{**many, "per": (1 << 24) - 1}) == NULL
    assert _reserve(window=0, table=None, **many) == NULL
