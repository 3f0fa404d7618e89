"""GPU: a server's steps as they follow one another - pages reserved, Q and K turned, rows cached, attended to - against
float64 all along."""

import numpy as np
import pytest
import torch

from oracle.pages import reserve
from oracle.paged import mx_values, paged_decode
from oracle.rotary import rotary
from test_gpu_mxfp4 import E2M1, _check_decode, _host
from test_gpu_paged import _gen

pytestmark = pytest.mark.gpu

I32 = torch.int32


def _tm():
    import paper_2608_17336_amd as tm
    return tm


class Model:
    """One attention layer's inputs: fused Q, K, V rows by (request, token)."""

    def __init__(self, Hq, Hk, d, dtype):
        self.Hq, self.Hk, self.d, self.dtype = Hq, Hk, d, dtype

    def rows(self, request, lo, hi):
        x = torch.randn(400, self.Hq + 2 * self.Hk, self.d, generator=_gen(5000 + request))
        return x[lo:hi].to(self.dtype)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("window", [0, 48])
@pytest.mark.parametrize("graph", [False, True])
def test_serve(dtype, window, graph):
    tm = _tm()
    B, Hq, Hk, d, page, per, P = 5, 8, 2, 64, 16, 24, 60
    layout, r = ("half", 64) if window else ("interleaved", 32)
    model = Model(Hq, Hk, d, dtype)
    f, g = tm.tilemix_rotary_frequencies(r, scaling="yarn", factor=4.0, original_len=100)
    cache = tm.PagedCache(*(t.view(torch.uint8).zero_().view(t.dtype) for t in tm.PagedCache.empty(P, page, Hk, d, E2M1)))
    free = tm.PageList.full(P)
    table, lens = torch.full((B, per), -1, dtype=I32, device="cuda"), torch.zeros(B, dtype=I32, device="cuda")
    first = torch.zeros(B, dtype=I32, device="cuda") if window else None
    want = torch.zeros(B, dtype=I32, device="cuda")
    room = 600                                                       # rows of a step, padded
    X = torch.zeros(room, Hq + 2 * Hk, d, dtype=dtype, device="cuda")
    Q, K, V = X[:, :Hq], X[:, Hq:Hq + Hk], X[:, Hq + Hk:]
    cu, pos, slots = (torch.zeros(n, dtype=t, device="cuda") for n, t in ((B + 1, I32), (room, I32), (room, torch.int64)))
    last = torch.zeros(B, 1, Hq, d, dtype=dtype, device="cuda")
    O, lse = torch.zeros_like(last), torch.zeros(B, Hq, device="cuda")
    ws = torch.empty(tm.tilemix_paged_decode_workspace_size(cache, table, lens, Hq) + 256, dtype=torch.uint8, device="cuda")

    def step():
        s = torch.cuda.current_stream()
        tm.tilemix_paged_reserve(free, table, lens, want, page, window=window, first_held=first, total=room, cu_seqlens=cu,
                                 positions=pos, slots=slots, stream=s)
        tm.tilemix_rotary(Q, K, f, pos, layout=layout, magnitude=g, Q_out=Q, K_out=K, stream=s)
        tm.tilemix_paged_append(cache, K, V, table, lens, cu, room, stream=s)
        last.copy_(Q[(cu[1:] - 1).clamp(min=0).long()][:, None])     # the last row of each sequence
        tm.tilemix_paged_decode(cache, last, table, lens, window=window, O=O, lse=lse, return_lse=True, workspace=ws, stream=s)

    run = step
    if graph:
        step()                                                       # (nothing is wanted yet)
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            step()
        run = captured.replay
    requests = [0, 1, 2, 3, 4]
    o = dict(table=[[-1] * per] * B, ids=list(range(P)), head=0, count=P, seqlens=[0] * B, first=[0] * B)
    script = [[33, 1, 0, 100, 16], [34, 2, 90, 101, 17], [35, 3, 91, 0, 18], [36, 3, 92, 60, 18 + 70], [37, 4, 0, 61, 89],
              [200, 5, 384, 62, 90], [201, 6, 30, 63, 0], [202, 200, 31, 64, 12]]
    for want_now in script:
        for b in range(B):
            if want_now[b] and not o["seqlens"][b]:
                requests[b] += 10                                    # a new request
        old = o["seqlens"]
        o = reserve(o["table"], old, want_now, page, o["ids"], o["head"], o["count"], window, o["first"], room)
        rows = [model.rows(requests[b], old[b], o["seqlens"][b]) for b in range(B)]
        x = torch.cat([t for t in rows if len(t)]) if any(len(t) for t in rows) else X[:0].cpu()
        assert len(x) <= room
        X.fill_(7.0)
        X[:len(x)] = x.cuda()
        want.copy_(torch.tensor(want_now, dtype=I32))
        O.fill_(float("nan"))
        run()
        torch.cuda.synchronize()
        assert lens.tolist() == o["seqlens"] and table.tolist() == o["table"] and free.state.tolist() == [o["head"], o["count"], o["refused"], 0]
        assert cu.tolist() == o["cu_seqlens"] and pos.tolist() == o["positions"] and slots.tolist() == o["slots"]
        assert (X[len(x):] == 7.0).all()                             # rows behind the last: as they were
        # What the cache holds at the slots, and what attention makes of it.
        host = _host(cache)
        k, v = (mx_values(host[i].numpy(), host[i + 2].numpy()) for i in (0, 1))
        turned = rotary(x[:, :Hq + Hk].double().numpy(), np.array(o["positions"][:len(x)]), f.cpu().numpy(), layout, g)
        for i, slot in enumerate(o["slots"][:len(x)]):
            if slot >= 0:
                # Half a step of E2M1, and one more where a rounding before tips it over: 2^e, with 2^e <= 2 a / 7.
                for got, w in ((k, turned[i, Hq:]), (v, x[i, Hq + Hk:].double().numpy())):
                    a = np.repeat(np.abs(w).reshape(Hk, d // 32, 32).max(-1), 32, -1)
                    assert (np.abs(got[slot // page, :, slot % page] - w) <= a * 2 / 7 * (2 + 2.0 ** -7)).all()
        q = last.double().cpu().numpy()[:, 0]
        ref = paged_decode(q, k, v, o["seqlens"], np.array(o["table"]), d ** -0.5, window)
        _check_decode(f"serve {want_now}", O, lse, ref, {torch.float16: "fp16", torch.bfloat16: "bf16"}[dtype], max(o["seqlens"]), v)
