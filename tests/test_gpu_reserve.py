"""GPU: pages for new tokens - every table, list, length, position and slot against the oracle."""

import random

import pytest
import torch

from oracle.pages import reserve

pytestmark = pytest.mark.gpu

I32 = torch.int32


def _tm():
    import paper_2608_17336_amd as tm
    return tm


def _gpu(x, dtype=I32):
    return torch.tensor(x, dtype=dtype).cuda()


class Server:
    """The state of a batch, on the GPU and in the oracle."""

    def __init__(self, B, per, page, P, window=0, capacity=None, head=0, seed=0):
        self.tm, self.page, self.window = _tm(), page, window
        order = list(range(P))
        random.Random(seed).shuffle(order)
        N = capacity or P
        ids = [-5] * N
        for i, p in enumerate(order):
            ids[(head + i) % N] = p
        self.table, self.lens, self.first, self.ids, self.head, self.count = [[-1] * per for _ in range(B)], [0] * B, [0] * B, ids, head, P
        self.list = self.tm.PageList(_gpu(ids), _gpu([head, P, 0, 0]))
        self.t, self.l, self.f = _gpu(self.table), _gpu(self.lens), _gpu(self.first) if window else None

    def step(self, want, total=None, stream=None):
        got = self.tm.tilemix_paged_reserve(self.list, self.t, self.l, _gpu(want), self.page, window=self.window, first_held=self.f,
                                            total=total, stream=stream)
        assert got.seqlens is self.l
        torch.cuda.synchronize()
        self.check(got, want, total)
        return got

    def check(self, got, want, total):
        w = reserve(self.table, self.lens, want, self.page, self.ids, self.head, self.count, self.window, self.first, total or 0)
        self.table, self.lens, self.first, self.ids, self.head, self.count = (w[k] for k in ("table", "seqlens", "first", "ids", "head", "count"))
        assert self.list.state.tolist() == [w["head"], w["count"], w["refused"], 0]
        assert self.l.tolist() == w["seqlens"] and got.cu_seqlens.tolist() == w["cu_seqlens"]
        assert self.t.tolist() == w["table"] and self.list.ids.tolist() == w["ids"]
        if self.window:
            assert self.f.tolist() == w["first"]
        if total is None:
            assert got.positions is None and got.slots is None
        else:
            assert got.positions.tolist() == w["positions"] and got.slots.tolist() == w["slots"]


@pytest.mark.parametrize("B,per,page,P", [(1, 1, 16, 1), (1, 9, 16, 5), (6, 9, 16, 40), (64, 12, 64, 500), (256, 5, 32, 700),
                                          (257, 5, 32, 700), (1024, 4, 16, 3000), (2500, 3, 256, 4000)])
@pytest.mark.parametrize("window", [0, 40])
def test_random_steps(B, per, page, P, window):
    """Sequences that begin, grow by one or many, stay, shorten, end, ask for too much; the ring wraps."""
    s = Server(B, per, page, P, window, capacity=P + 3, head=P // 2, seed=B)
    rng = random.Random(B + window)
    for i in range(12 if B < 1000 else 5):
        want = [rng.choice([0, n, n + 1, n + 1, n + 1, n + rng.randrange(1, 3 * page), max(0, n - rng.randrange(page)), per * page,
                            per * page + 1]) for n in s.lens]
        if i % 4 == 3:
            want = [0 if rng.random() < 0.7 else n + 1 for n in s.lens]
        new = sum(max(0, w - n) for w, n in zip(want, s.lens))
        s.step(want, total=rng.choice([None, 0, new, new + 9, new // 2]))


def test_prompts_over_many_workgroups():
    """Entries and rows shared by many workgroups, sequences without any among them."""
    B, per, page = 100, 700, 16
    s = Server(B, per, page, 30000, head=29990)
    want = [(0, 1, 5000, 16, 11200, 333)[b * b % 6] for b in range(B)]
    s.step(want, total=sum(want) + 1000)
    s.step([0 if b % 3 else n + 700 for b, n in enumerate(s.lens)], total=90000)


def test_state_and_lengths_beside_the_old():
    """With state_out and seqlens_out nothing of the old state changes but the table and the ring behind its end, and
    the same call again gives the same."""
    tm = _tm()
    s = Server(5, 8, 16, 30, capacity=64, head=60)
    s.step([16, 33, 1, 0, 100])
    want = _gpu([17, 0, 1, 40, 128])
    before = (s.list.state.clone(), s.l.clone())
    outs = []
    for _ in range(2):
        new = (torch.full((4,), 99, dtype=I32, device="cuda"), torch.full((5,), 99, dtype=I32, device="cuda"))
        cu, pos, slots = torch.empty(6, dtype=I32, device="cuda"), torch.empty(80, dtype=I32, device="cuda"), torch.empty(80, dtype=torch.int64, device="cuda")
        got = tm.tilemix_paged_reserve(s.list, s.t, s.l, want, 16, total=80, state_out=new[0], seqlens_out=new[1], cu_seqlens=cu,
                                       positions=pos, slots=slots)
        assert got.seqlens is new[1] and got.cu_seqlens is cu and got.positions is pos and got.slots is slots
        torch.cuda.synchronize()
        assert torch.equal(s.list.state, before[0]) and torch.equal(s.l, before[1])
        if not outs:
            kept = s.t.clone()
            kept[1] = _gpu(s.table[1])         # (given back: -1 now, and read again)
            s.t.copy_(kept)
        outs.append([x.clone() for x in (*new, cu, pos, slots, s.list.ids)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    s.list = tm.PageList(s.list.ids, new[0])
    s.l = new[1]
    s.check(got, want.tolist(), 80)


@pytest.mark.parametrize("want,P", [([2 ** 31 - 1] * 7, 40), ([2 ** 30] * 9, 3), ([-5, -2 ** 31, 3], 4)])
def test_extreme_lengths(want, P):
    """Sums beyond 32 bits, lengths past the page table, negative ones; a page table of 2^26 entries whose rows overlap nothing
    that is written."""
    per = 12
    s = Server(len(want), per, 16, P)
    s.step(want, total=20)
    s.step([5] * len(want), total=50)
    # The table's rows are the first entries of long ones: requests that no list can serve.
    tm = _tm()
    state, ids = _gpu([0, P, 0, 0]), _gpu(list(range(P)))
    B = len(want)
    wide = torch.full((B, 1 << 20), -1, dtype=I32, device="cuda")
    lens = torch.zeros(B, dtype=I32, device="cuda")
    got = tm.tilemix_paged_reserve(tm.PageList(ids, state), wide, lens, _gpu([1 << 24] * B), 16)
    assert state.tolist() == [0, P, B, 0] and not lens.any() and (wide == -1).all() and not got.cu_seqlens.any()


def test_sums_that_pass_32_bits():
    """65535 sequences that together want 2^43 tokens: the first is served, the others refused."""
    tm = _tm()
    B = 65535
    state, ids = _gpu([0, 8, 0, 0]), _gpu(list(range(8)))
    table = torch.full((B, 64), -1, dtype=I32, device="cuda")
    lens, want = torch.zeros(B, dtype=I32, device="cuda"), torch.full((B,), 128, dtype=I32, device="cuda")
    want[1:] = 64 * 256
    long = tm.tilemix_paged_reserve(tm.PageList(ids, state), table, lens, want, 16 * 16, total=200)
    assert state.tolist() == [1, 7, B - 1, 0] and lens[0] == 128 and not lens[1:].any()
    assert long.cu_seqlens[0] == 0 and (long.cu_seqlens[1:] == 128).all()
    assert long.positions.tolist() == list(range(128)) + [-1] * 72 and long.slots.tolist() == list(range(128)) + [-1] * 72
    # With a window rows need few pages: their sum stops at 2^30 - 1.
    state = _gpu([0, 8, 0, 0])
    table.fill_(-1)
    lens, first = torch.zeros(4, dtype=I32, device="cuda"), torch.zeros(4, dtype=I32, device="cuda")
    wide = torch.full((4, 1 << 22), -1, dtype=I32, device="cuda")
    got = tm.tilemix_paged_reserve(tm.PageList(ids, state), wide, lens, _gpu([2 ** 30 - 256] * 4), 256, window=256, first_held=first, total=0)
    assert state.tolist() == [4, 4, 0, 0] and (lens == 2 ** 30 - 256).all()
    assert got.cu_seqlens.tolist() == [0, 2 ** 30 - 256, 2 ** 30 - 1, 2 ** 30 - 1, 2 ** 30 - 1]
    assert (wide.sum(1) == torch.arange(4, device="cuda") - (2 ** 22 - 1)).all() and first.tolist() == [2 ** 22 - 2] * 4


def test_broken_state_stays_in_bounds():
    """A head and a count outside the list, lengths outside the table: clamped."""
    tm = _tm()
    guard = torch.full((20,), 7, dtype=I32, device="cuda")
    ids = guard[5:10]
    ids.copy_(torch.arange(5))
    for head, count in ((2 ** 31 - 1, 2 ** 31 - 1), (-3, -1), (7, 100)):
        table = torch.full((4, 6), -1, dtype=I32, device="cuda")
        lens = _gpu([-9, 2 ** 31 - 1, 0])
        state = _gpu([head, count, 0, 0])
        tm.tilemix_paged_reserve(tm.PageList(ids, state), table[:3], lens, _gpu([16, 3, 40]), 16, total=30)
        torch.cuda.synchronize()
        assert (guard[:5] == 7).all() and (guard[10:] == 7).all() and (table[3] == -1).all()
        assert 0 <= state[0] < 5 and 0 <= state[1] <= 5 and lens[1] == 3


def test_a_table_that_is_a_slice_and_another_stream():
    s = Server(4, 6, 16, 30)
    wide = torch.full((4, 11), -7, dtype=I32, device="cuda")
    wide[:, :6] = -1
    s.t = wide[:, :6]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.step([3, 90, 0, 17], total=120, stream=side)
    s.step([3, 0, 50, 18], total=60, stream=side)
    assert (wide[:, 6:] == -7).all()


@pytest.mark.parametrize("window", [0, 24])
def test_captured_in_a_graph(window):
    """Every replay takes the lengths and state of its time, with other work between."""
    B, per, page, total = 40, 20, 16, 900
    s = Server(B, per, page, 300, window, seed=5)
    s.step([b % 50 for b in range(B)])
    want, cu = torch.zeros(B, dtype=I32, device="cuda"), torch.zeros(B + 1, dtype=I32, device="cuda")
    pos, slots = torch.zeros(total, dtype=I32, device="cuda"), torch.zeros(total, dtype=torch.int64, device="cuda")

    def call():
        return s.tm.tilemix_paged_reserve(s.list, s.t, s.l, want, page, window=window, first_held=s.f, total=total, cu_seqlens=cu,
                                          positions=pos, slots=slots, stream=torch.cuda.current_stream())

    want.copy_(s.l)
    call()
    s.check(call(), s.lens, total)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    rng = random.Random(6)
    for _ in range(5):
        new = [rng.choice([0, n + 1, n + 1, n + 40, n]) for n in s.lens]
        want.copy_(_gpu(new))
        pos.fill_(77), slots.fill_(77), cu.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        s.check(got, new, total)


@pytest.mark.parametrize("B,rows", [(3, 40), (200, 2000), (1500, 300)])
def test_lengths_written_over_the_wanted_ones(B, rows):
    """seqlens_out may be `wanted`, which all workgroups read, and seqlens itself may be what is wanted."""
    tm = _tm()
    rng = random.Random(B)
    for _ in range(3):
        old, want = [rng.randrange(rows) for _ in range(B)], [rng.randrange(2 * rows) for _ in range(B)]
        per, P = -(-2 * rows // 16), B * (2 * rows // 16 + 2)
        s = Server(B, per, 16, P, seed=1)
        s.step(old)
        w = _gpu(want)
        state = torch.empty(4, dtype=I32, device="cuda")
        total = sum(max(0, n - o) for o, n in zip(old, want))
        got = tm.tilemix_paged_reserve(s.list, s.t, s.l, w, 16, total=total, state_out=state, seqlens_out=w)
        torch.cuda.synchronize()
        assert got.seqlens is w and s.l.tolist() == old
        s.list, s.l = tm.PageList(s.list.ids, state), w
        s.check(got, want, total)
        got = tm.tilemix_paged_reserve(s.list, s.t, s.l, s.l, 16, total=5)
        s.check(got, want, 5)


def test_binding_refusals():
    tm = _tm()
    s = Server(2, 3, 16, 4)
    want = _gpu([1, 1])
    ok = (s.list, s.t, s.l, want, 16)
    for bad, kw in (((s.list, s.t, s.l, want.long(), 16), {}), ((s.list, s.t[0], s.l, want, 16), {}), (ok, dict(window=3)),
                    (ok, dict(first_held=s.l.clone())), (ok, dict(positions=want)), (ok, dict(total=5, positions=want)),
                    (ok, dict(total=2, slots=want)), (ok, dict(state_out=want)), (ok, dict(total=-1)), (ok, dict(seqlens_out=want.cpu())),
                    ((tm.PageList(s.list.ids, want), *ok[1:]), {}), ((*ok[:4], 2 ** 32 + 16), {}), ((*ok[:4], 24), {}),
                    ((s.list, s.t.T, s.l, want, 16), {})):
        with pytest.raises((ValueError, TypeError, tm.TilemixError)):
            tm.tilemix_paged_reserve(*bad, **kw)
    torch.cuda.synchronize()
    assert s.list.state.tolist() == [0, 4, 0, 0] and (s.t == -1).all()
