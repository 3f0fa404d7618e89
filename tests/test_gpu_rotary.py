"""GPU: rotary positions against float64."""

from fractions import Fraction

import numpy as np
import pytest
import torch

from gpu_util import log
from oracle.rotary import frequencies, rotary

pytestmark = pytest.mark.gpu

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
LAYOUTS = ["half", "interleaved"]


def _tm():
    import paper_2608_17336_amd as tm
    return tm


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _x(shape, dtype, seed, gain=1.0):
    return (torch.randn(shape, generator=_gen(seed)) * gain).to(TYPES[dtype])


def _check(name, got, x, pos, f, layout, dtype, g=1.0, inverse=False):
    """Half a step of the type, and FP32: a cosine or sine is off by at most 4 2^-24 (its argument by 2^-24 and its
    factor pi / 2 by 2^-25 of at most 0.8, the last sums by two roundings) and, of its FP64 angle and the oracle's, by
    2^-51 of the angle; its product with g and x, and their sum, add two roundings to each term: 8 2^-24 of
    g (|x1| + |x2|) in all.  Channels that do not turn are equal."""
    want = rotary(x.double().numpy(), pos, f, layout, g, inverse)
    r = 2 * len(f)
    mass = rotary(x.double().abs().numpy(), np.zeros(len(pos)), np.zeros_like(f), layout)
    a, b = (np.arange(r // 2), np.arange(r // 2) + r // 2) if layout == "half" else (2 * np.arange(r // 2), 2 * np.arange(r // 2) + 1)
    both = mass[..., a] + mass[..., b]
    off = 8 * 2.0 ** -24 + 2.0 ** -51 * np.abs(pos.astype(np.float64)[:, None] * f)[:, None]
    tol = np.zeros_like(want)
    tol[..., a] = tol[..., b] = abs(g) * both * off
    fi = torch.finfo(TYPES[dtype])
    tol += fi.eps / 2 * np.abs(want) + fi.smallest_normal * fi.eps
    err = np.abs(got.double().cpu().numpy() - want)
    log(f"rotary {name}: error/tolerance {(err / tol).max() if err.size else 0:.3f}")
    assert (err <= tol).all(), name
    assert torch.equal(got.cpu()[..., r:].view(torch.int16), x[..., r:].contiguous().view(torch.int16)), name


def _positions(n, seed, top=200000):
    pos = torch.randint(0, top, (n,), generator=_gen(seed), dtype=torch.int32)
    pos[: min(n, 3)] = torch.tensor([0, 1, 131071], dtype=torch.int32)[: min(n, 3)]
    return pos


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("d,r", [(64, 64), (64, 32), (64, 2), (64, 24), (64, 62), (128, 128), (128, 64), (128, 96), (128, 80), (128, 30),
                                 (128, 44), (128, 126)])
@pytest.mark.parametrize("n,Hq,Hk", [(1, 2, 2), (13, 28, 4), (37, 5, 1)])
def test_every_part_of_a_head(dtype, layout, d, r, n, Hq, Hk):
    """Rotary parts whose halves are aligned to 16, 8, 4 and 2 bytes; heads that fill a workgroup and that do not."""
    tm = _tm()
    Q, K, pos = _x((n, Hq, d), dtype, 1), _x((n, Hk, d), dtype, 2), _positions(n, 3)
    f, _ = tm.tilemix_rotary_frequencies(r)
    for inverse in (False, True):
        q, k = tm.tilemix_rotary(Q.cuda(), K.cuda(), f, pos.cuda(), layout=layout, magnitude=1.25, inverse=inverse)
        for got, x in ((q, Q), (k, K)):
            assert got.dtype == x.dtype and got.shape == x.shape
            _check(f"{dtype} {layout} d{d} r{r} n{n}", got, x, pos.numpy(), f.cpu().numpy(), layout, dtype, 1.25, inverse)
    qi, ki = Q.cuda(), K.cuda()
    got = tm.tilemix_rotary(qi, ki, f, pos.cuda(), layout=layout, magnitude=1.25, inverse=True, Q_out=qi, K_out=ki)
    assert got[0] is qi and got[1] is ki and torch.equal(qi, q) and torch.equal(ki, k)   # in place
    qi = Q.cuda()
    q1, k1 = tm.tilemix_rotary(qi, K.cuda(), f, pos.cuda(), layout=layout, magnitude=1.25, inverse=True, Q_out=qi)
    assert torch.equal(q1, q) and torch.equal(k1, k)                                     # one of them


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_many_rows(dtype, layout):
    """Workgroups of several tokens, the last of them not full."""
    tm = _tm()
    for n, Hq, Hk, d, r in ((9001, 2, 1, 64, 64), (5003, 8, 8, 128, 64), (4099, 3, 0, 64, 20)):
        Q, K, pos = _x((n, Hq, d), dtype, 10), _x((n, Hk, d), dtype, 11) if Hk else None, _positions(n, 12)
        f, _ = tm.tilemix_rotary_frequencies(r)
        got = tm.tilemix_rotary(Q.cuda(), None if K is None else K.cuda(), f, pos.cuda(), layout=layout)
        for y, x in zip(got, (Q, K)):
            if x is not None:
                _check(f"{n} rows {dtype} {layout}", y, x, pos.numpy(), f.cpu().numpy(), layout, dtype)
        assert (got[1] is None) == (K is None)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_positions(layout):
    """Angles whose FP32 product would be off by whole turns."""
    tm = _tm()
    pos = torch.tensor([2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30 + 1, 2 ** 24 + 1, 10 ** 6 + 1, 2 ** 20, 131073], dtype=torch.int32)
    Q = _x((7, 2, 64), "fp16", 20)
    for kw in (dict(), dict(scaling="yarn", factor=32.0, original_len=4096), dict(scaling="ntk", factor=8.0)):
        f, g = tm.tilemix_rotary_frequencies(64, **kw)
        q, _ = tm.tilemix_rotary(Q.cuda(), None, f, pos.cuda(), layout=layout, magnitude=g)
        _check(f"far {kw}", q, Q, pos.numpy(), f.cpu().numpy(), layout, "fp16", g)


def _pi(bits=400):
    """pi 2^bits as a whole number: 16 arctan(1/5) - 4 arctan(1/239)."""
    def arctan(x):
        t = (1 << (bits + 32)) // x
        total, n = t, 1
        while t:
            t //= -x * x
            n += 2
            total += t // n
        return total
    return (16 * arctan(5) - 4 * arctan(239)) >> 32


def _exact_cos_sin(p, f):
    """cos(p f) and sin(p f), from the angle's remainder by a quarter turn in whole numbers."""
    num, den = float(f).as_integer_ratio()           # den: a power of two
    quarter = _pi() * den >> 1                       # 2^400 den pi / 2
    k, rest = divmod((p * num << 400) + quarter // 2, quarter)
    a = float(Fraction(rest - quarter // 2, den << 400))
    c, s = np.cos(a), np.sin(a)
    return ((c, s), (-s, c), (-c, -s), (s, -c))[k % 4]


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_angles_next_to_quarter_turns(layout):
    """(1, 0) turned by angles of positions up to 2^31 whose cosine is next to 0: the BF16 result has its own size's bits, and
    shows what the angle has lost.  A cosine or sine is off by 8 2^-24 of itself (the argument's 2^-24 and its factor's 2^-25, the
    last sums' roundings) and the FP64 angle's 2^-52 of a turn, below 2^-48; the result rounds by half a step."""
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(128)
    host = f.cpu().numpy()
    pos = []
    for i in (0, 1, 2, 7, 20, 40):
        k = np.arange(1 << 21) + int((2 ** 31 - 10) * host[i] / np.pi) - (1 << 21)
        k = k[k >= 0]
        p = np.rint((k + 0.5) * np.pi / host[i])
        near = np.abs(p * host[i] - (k + 0.5) * np.pi) < 1e-5
        pos += p[near & (p < 2 ** 31)].astype(int).tolist()[-40:]
    assert len(pos) > 100
    x = torch.zeros(len(pos), 1, 128)
    x[..., :64] = 1.0
    if layout == "interleaved":
        x = x.view(-1, 1, 2, 64).transpose(2, 3).reshape(-1, 1, 128)
    q, _ = tm.tilemix_rotary(x.bfloat16().cuda(), None, f, torch.tensor(pos, dtype=torch.int32).cuda(), layout=layout)
    got = q.double().cpu().numpy()[:, 0]
    got = (got[:, :64], got[:, 64:]) if layout == "half" else (got[:, 0::2], got[:, 1::2])
    want = np.array([[_exact_cos_sin(p, v) for v in host] for p in pos])
    assert (np.abs(want[..., 0]) < 1e-5).sum() > 100
    for j in range(2):
        err, tol = np.abs(got[j] - want[..., j]), np.abs(want[..., j]) * (2.0 ** -8 + 2.0 ** -21) + 2.0 ** -48
        log(f"rotary next to quarter turns {layout} {j}: error/tolerance {(err / tol).max():.3f}")
        assert (err <= tol).all(), (err / tol).max()


def test_every_angle_of_a_turn():
    """One pair that turns by n / 4096 of a turn: cosines and sines to 2^-22, through BF16's whole range of sizes of x."""
    tm = _tm()
    n = 4096
    f = torch.tensor([2 * np.pi / n] + [0.0] * 31, dtype=torch.float64, device="cuda")
    pos = torch.arange(n, dtype=torch.int32)
    for e in (-120, -20, 0, 60, 126):
        x = torch.zeros(n, 1, 64)
        x[:, 0, 0], x[:, 0, 32] = 2.0 ** e, 0.0
        x[::2, 0, 32], x[::2, 0, 0] = 2.0 ** e, 0.0
        x = x.bfloat16()
        q, _ = tm.tilemix_rotary(x.cuda(), None, f, pos.cuda())
        _check(f"angles 2^{e}", q, x, pos.numpy(), f.cpu().numpy(), "half", "bf16")


def _packed(new, lens):
    """Positions of packed rows."""
    return torch.cat([torch.arange(n - m, n, dtype=torch.int32) for m, n in zip(new, lens)])


@pytest.mark.parametrize("B", [1, 3, 64, 65, 150, 5000])
def test_positions_from_lengths(B):
    """The last rows of sequences: packed, with empty ones at both ends and in runs; and L of each."""
    tm = _tm()
    new = [(0, 1, 7, 0, 0, 3)[(b * b + 1) % 6] if B > 3 else (0, 40, 1)[b % 3] + (B == 1) for b in range(B)]
    lens = [n + (b * 37) % 1000 for b, n in enumerate(new)]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32)
    total = int(cu[-1])
    Q, K = _x((total + 5, 4, 64), "bf16", 30), _x((total + 5, 2, 64), "bf16", 31)    # five rows that no sequence owns
    f, _ = tm.tilemix_rotary_frequencies(64)
    l_gpu = torch.tensor(lens, dtype=torch.int32).cuda()
    out = [torch.full_like(x, 9.0).cuda() for x in (Q, K)]
    got = tm.tilemix_rotary(Q.cuda(), K.cuda(), f, seqlens_k=l_gpu, cu_seqlens=cu.cuda(), Q_out=out[0], K_out=out[1])
    pos = _packed(new, lens)
    want = tm.tilemix_rotary(Q[:total].cuda(), K[:total].cuda(), f, pos.cuda())
    for y, w, x in zip(got, want, (Q, K)):
        assert torch.equal(y[:total], w) and (y[total:] == 9.0).all()
        _check(f"packed B {B}", w, x[:total], pos.numpy(), f.cpu().numpy(), "half", "bf16")
    for L in (1, 3):
        Q = _x((B, L, 4, 64), "fp16", 32)
        q, _ = tm.tilemix_rotary(Q.cuda(), None, f, seqlens_k=l_gpu + L)
        pos = (torch.tensor(lens)[:, None] + torch.arange(L)).to(torch.int32)
        w, _ = tm.tilemix_rotary(Q.cuda(), None, f, pos.cuda())
        assert torch.equal(q, w)
        _check(f"padded B {B} L {L}", w.flatten(0, 1), Q.flatten(0, 1), pos.flatten().numpy(), f.cpu().numpy(), "half", "fp16")


def test_rows_without_a_position():
    """Negative positions, lengths shorter than the rows, broken offsets: those rows stay as they were, and no row beyond
    the last is touched."""
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(64)
    Q = _x((8, 2, 64), "fp16", 40)
    pos = torch.tensor([5, -1, 7, -2 ** 31, 0, -7, 9, 1], dtype=torch.int32)
    out = torch.full((10, 2, 64), 3.0, dtype=torch.float16, device="cuda")
    tm.tilemix_rotary(Q.cuda(), None, f, pos.cuda(), Q_out=out[:8])
    ok = pos >= 0
    assert (out[:8][~ok.cuda()] == 3.0).all() and (out[8:] == 3.0).all()
    _check("some positions", out[:8][ok.cuda()], Q[ok], pos[ok].numpy(), f.cpu().numpy(), "half", "fp16")
    out.fill_(3.0)
    Q4 = Q.view(2, 4, 2, 64)
    tm.tilemix_rotary(Q4.cuda(), None, f, seqlens_k=torch.tensor([2, 100], dtype=torch.int32).cuda(), Q_out=out[:8].view(2, 4, 2, 64))
    assert (out[:2] == 3.0).all() and (out[8:] == 3.0).all()
    _check("short sequence", out[2:8], Q[2:], np.array([0, 1, 96, 97, 98, 99]), f.cpu().numpy(), "half", "fp16")
    for cu in ([-5, 4, 3, 2 ** 31 - 1], [6, 2, 2, 1], [0, -2 ** 31, 9, 8]):
        out.fill_(3.0)
        tm.tilemix_rotary(Q.cuda(), None, f, seqlens_k=torch.tensor([30, 30, 30], dtype=torch.int32).cuda(),
                          cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), Q_out=out[:8])
        assert (out[8:] == 3.0).all()


@pytest.mark.parametrize("layout", LAYOUTS)
def test_slices_of_a_fused_projection(layout):
    """Q and K side by side with V, read and written in place; dense outputs; [B, L] rows and one row a sequence; one
    row for all."""
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(96)
    for shape in ((21,), (3, 7), (5, 1)):
        X = _x((*shape, 8 + 2 + 2, 128), "fp16", 50)
        pos = _positions(X[..., 0, 0].numel(), 51).view(shape)
        Q, K = X[..., :8, :], X[..., 8:10, :]
        g = X.cuda()
        q, k = tm.tilemix_rotary(g[..., :8, :], g[..., 8:10, :], f, pos.cuda(), layout=layout)
        for y, x in ((q, Q), (k, K)):
            assert y.is_contiguous()
            _check(f"slices {shape}", y.reshape(-1, *y.shape[-2:]), x.reshape(-1, *x.shape[-2:]), pos.flatten().numpy(), f.cpu().numpy(),
                   layout, "fp16")
        tm.tilemix_rotary(g[..., :8, :], g[..., 8:10, :], f, pos.cuda(), layout=layout, Q_out=g[..., :8, :], K_out=g[..., 8:10, :])
        assert torch.equal(g[..., :8, :], q) and torch.equal(g[..., 8:10, :], k) and torch.equal(g[..., 10:, :].cpu(), X[..., 10:, :])
    one = _x((1, 4, 128), "fp16", 52).cuda()
    pos = _positions(6, 53).cuda()
    a, _ = tm.tilemix_rotary(one.expand(6, 4, 128), None, f, pos, layout=layout)
    b, _ = tm.tilemix_rotary(one.expand(6, 4, 128).contiguous(), None, f, pos, layout=layout)
    assert torch.equal(a, b)


def test_what_does_not_turn_is_moved_as_it_is():
    """Infinities and NaN behind rotary_dim, with their payloads; in front of it they stay in their pair."""
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(32)
    for layout in LAYOUTS:
        x = _x((3, 1, 64), "fp16", 60)
        x.view(torch.int16)[1, 0, 40] = 0x7c01
        x[1, 0, 50] = float("inf")
        x[2, 0, 3] = float("nan")
        y, _ = tm.tilemix_rotary(x.cuda(), None, f, torch.tensor([3, 4, 5], dtype=torch.int32).cuda(), layout=layout)
        y = y.cpu()
        assert torch.equal(y[..., 32:].view(torch.int16), x[..., 32:].contiguous().view(torch.int16))
        bad = torch.isnan(y[2, 0]).nonzero().flatten().tolist()
        assert bad == ([3, 19] if layout == "half" else [2, 3]) and not torch.isnan(y[0]).any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_gradient(dtype, layout):
    """<w, rotary(x)> against <rotary^-1(w), x>, and differences of the forward pass: the step 2^-3 of inputs on a grid of
    2^-3 is exact in both types."""
    tm = _tm()
    n, H, d, r = 9, 3, 64, 48
    f, _ = tm.tilemix_rotary_frequencies(r)
    pos = _positions(n, 70).cuda()
    x, w = ((torch.randint(-16, 17, (n, H, d), generator=_gen(71 + i)) / 8).to(TYPES[dtype]) for i in range(2))
    y, _ = tm.tilemix_rotary(x.cuda(), None, f, pos, layout=layout, magnitude=1.5)
    grad, _ = tm.tilemix_rotary(w.cuda(), None, f, pos, layout=layout, magnitude=1.5, inverse=True)
    y, grad, x, w = (t.cpu().double() for t in (y, grad, x, w))
    eps = torch.finfo(TYPES[dtype]).eps
    # Both sides are rounded: half a step of each output (|y|, |grad| <= 1.5 2 sqrt 2), and FP32's error far below.
    tol = (w.abs() * y.abs()).sum() * eps / 2 + (grad.abs() * x.abs()).sum() * eps / 2
    assert abs((w * y).sum() - (grad * x).sum()) <= tol * 1.01
    for c in (0, 5, 24, 47, 48, 63):
        step = torch.zeros(n, H, d, dtype=torch.float64)
        step[..., c] = 0.125
        up, _ = tm.tilemix_rotary((x + step).to(TYPES[dtype]).cuda(), None, f, pos, layout=layout, magnitude=1.5)
        down, _ = tm.tilemix_rotary((x - step).to(TYPES[dtype]).cuda(), None, f, pos, layout=layout, magnitude=1.5)
        up, down = up.cpu().double(), down.cpu().double()
        diff = (w * (up - down)).sum(-1) / 0.25
        # A channel reaches the two outputs of its pair; the others are equal.  Half a step of both, divided by the step.
        touched = (up != down)
        assert touched.sum(-1).max() <= 2
        tol = ((w.abs() * (up.abs() + down.abs()) * eps / 2 * touched).sum(-1) / 0.25 + grad[..., c].abs() * eps / 2) * 1.01 + 1e-6
        assert ((diff - grad[..., c]).abs() <= tol).all(), c


def test_streams_and_graph():
    """On a stream of its own, and captured: every replay takes the rows and positions of its time."""
    tm = _tm()
    B, Hq, Hk, d = 6, 8, 2, 128
    f, _ = tm.tilemix_rotary_frequencies(128)
    q, k = torch.zeros(B, 1, Hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, 1, Hk, d, dtype=torch.bfloat16, device="cuda")
    qo, ko, lens = torch.zeros_like(q), torch.zeros_like(k), torch.zeros(B, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = tm.tilemix_rotary(q, k, f, seqlens_k=lens + 5, stream=side)
    side.synchronize()
    assert not a[0].any()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tm.tilemix_rotary(q, k, f, seqlens_k=lens, Q_out=qo, K_out=ko, stream=torch.cuda.current_stream())
    for r in range(4):
        lens += 1000 * r + 1
        q.copy_(_x(q.shape, "bf16", 80 + r)), k.copy_(_x(k.shape, "bf16", 90 + r))
        qo.fill_(float("nan")), ko.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        w = tm.tilemix_rotary(q, k, f, seqlens_k=lens)
        assert torch.equal(qo, w[0]) and torch.equal(ko, w[1])
        _check("replay", qo[:, 0], q[:, 0].cpu(), lens.cpu().numpy() - 1, f.cpu().numpy(), "half", "bf16")


@pytest.mark.parametrize("layout", LAYOUTS)
def test_more_rows_than_the_caches_hold(layout):
    """More than 2^27 bytes of results at once, also in place, are those of several calls."""
    tm = _tm()
    n, Hq, Hk, d = 17001, 28, 4, 128
    assert n * (Hq + Hk) * d * 2 > 2 ** 27
    g = torch.Generator(device="cuda").manual_seed(97)
    q, k = (torch.randn(n, H, d, generator=g, device="cuda").half() for H in (Hq, Hk))
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 7
    for r in (128, 64, 8):
        f, _ = tm.tilemix_rotary_frequencies(r)
        a, b = tm.tilemix_rotary(q, k, f, pos, layout=layout)
        for lo in range(0, n, 4000):
            s = slice(lo, lo + 4000)
            x, y = tm.tilemix_rotary(q[s], k[s], f, pos[s], layout=layout)
            assert torch.equal(a[s], x) and torch.equal(b[s], y)
        qi, ki = q.clone(), k.clone()
        tm.tilemix_rotary(qi, ki, f, pos, layout=layout, Q_out=qi, K_out=ki)
        assert torch.equal(qi, a) and torch.equal(ki, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_results_past_the_caches(layout, dtype):
    """More than 2^28 bytes of results at once, also in place and of rows without a position, are those of several calls."""
    tm = _tm()
    n, Hq, Hk, d = 33001, 28, 4, 128
    assert n * (Hq + Hk) * d * 2 > 2 ** 28
    g = torch.Generator(device="cuda").manual_seed(99)
    q, k = (torch.randn(n, H, d, generator=g, device="cuda").to(TYPES[dtype]) for H in (Hq, Hk))
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 7
    pos[::11] = -1
    for r in (128, 48):
        f, _ = tm.tilemix_rotary_frequencies(r)
        out = [torch.full_like(t, 7) for t in (q, k)]
        tm.tilemix_rotary(q, k, f, pos, layout=layout, Q_out=out[0], K_out=out[1])
        assert all((t[::11] == 7).all() for t in out)
        for lo in range(0, n, 9000):
            s = slice(lo, lo + 9000)
            x, y = (torch.full_like(t[s], 7) for t in (q, k))
            tm.tilemix_rotary(q[s], k[s], f, pos[s], layout=layout, Q_out=x, K_out=y)
            assert torch.equal(out[0][s], x) and torch.equal(out[1][s], y)
        qi, ki = q.clone(), k.clone()
        tm.tilemix_rotary(qi, ki, f, pos, layout=layout, Q_out=qi, K_out=ki)
        moved = pos >= 0
        assert torch.equal(qi[moved], out[0][moved]) and torch.equal(ki[moved], out[1][moved])
        assert torch.equal(qi[~moved], q[~moved]) and torch.equal(ki[~moved], k[~moved])


def test_offsets_past_32_bits():
    """Rows 2^31 elements in, and rows that lie far apart."""
    tm = _tm()
    n, H, d = 2 ** 31 // (64 * 128) + 40, 64, 128
    f, _ = tm.tilemix_rotary_frequencies(128)
    x = torch.empty((n, H, d), dtype=torch.float16, device="cuda")
    x[-30:] = _x((30, H, d), "fp16", 95).cuda()
    pos = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    pos[-30:] = torch.arange(30, device="cuda") * 1001
    want, _ = tm.tilemix_rotary(x[-30:].contiguous(), None, f, pos[-30:].contiguous())
    apart = x.view(-1)[: 2 * (2 ** 30 + 1024)].view(2, -1)[:, : 4 * d].view(2, 4, d)      # two rows 2^30 elements apart
    apart.copy_(_x((2, 4, d), "fp16", 96).cuda())
    near, _ = tm.tilemix_rotary(apart, None, f, pos[-2:].contiguous())
    ref, _ = tm.tilemix_rotary(apart.contiguous(), None, f, pos[-2:].contiguous())
    assert torch.equal(near, ref)
    tm.tilemix_rotary(x, None, f, pos, Q_out=x)
    assert torch.equal(x[-30:], want)


def test_binding_refusals():
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(64)
    q, pos = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ok = dict(Q=q, K=None, inv_freq=f, positions=pos)
    cu = torch.tensor([0, 4], dtype=torch.int32).cuda()
    for kw in (dict(Q=q.float()), dict(Q=q[0]), dict(K=q.bfloat16()), dict(K=q[:3]), dict(inv_freq=f.float()), dict(inv_freq=f.cpu()),
               dict(inv_freq=torch.cat([f, f])), dict(positions=pos.long()), dict(positions=pos[:3]), dict(positions=None),
               dict(seqlens_k=pos), dict(positions=None, seqlens_k=pos), dict(positions=None, seqlens_k=pos, cu_seqlens=cu),
               dict(layout="both"), dict(magnitude=float("inf")), dict(Q_out=q[:3]), dict(Q_out=q.bfloat16()),
               dict(Q=q.transpose(0, 1)), dict(Q=torch.zeros(4, 2, 66, dtype=torch.float16, device="cuda")[..., :64]),
               dict(Q_out=torch.zeros(1, 2, 64, dtype=torch.float16, device="cuda").expand(4, 2, 64))):
        with pytest.raises((ValueError, TypeError, tm.TilemixError)):
            tm.tilemix_rotary(**{**ok, **kw})


def test_more_workgroups_than_a_launch_has_in_x():
    """2^27 rows of one head, 8 of them in a workgroup: 2^32 threads and more."""
    tm = _tm()
    n, d = 2 ** 27 + 5, 64
    f, _ = tm.tilemix_rotary_frequencies(d)
    at = torch.cat([torch.arange(a, b, device="cuda") for a, b in ((0, 20), (2 ** 26 - 11, 2 ** 26 + 13), (n - 25, n))])
    x, own = torch.empty((n, 1, d), dtype=torch.float16, device="cuda"), _x((len(at), 1, d), "fp16", 97).cuda()
    x[at] = own
    pos, some = torch.full((n,), -1, dtype=torch.int32, device="cuda"), _positions(len(at), 98).cuda()
    pos[at] = some
    want, _ = tm.tilemix_rotary(own, None, f, some)
    tm.tilemix_rotary(x, None, f, pos, Q_out=x)
    assert torch.equal(x[at], want)


def test_k_out_goes_with_k():
    tm = _tm()
    f, _ = tm.tilemix_rotary_frequencies(64)
    q, pos = torch.zeros(4, 2, 64, dtype=torch.float16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        tm.tilemix_rotary(q, None, f, pos, K_out=torch.empty_like(q))
