"""Timed cases of the paged key/value cache: writing it, reading it back, attending to it.

A pool holds pages of ``page`` token slots, K and V [pages, Hk, page, d], in FP16, BF16, INT8 or
E4M3; the 8-bit formats have one FP32 scale per row (a token's d channels of one head).  A page
table [B, max_pages] and lengths [B] say which slots hold the tokens of each sequence.

  append   tilemix_paged_append: new rows become the last rows of their sequences.  8-bit formats are
           read back by tilemix_paged_gather, so that the outputs are the values that the codes
           stand for; 16-bit formats return the pool itself.
  gather   tilemix_paged_gather: the rows of every sequence, packed and in 16 bits
  decode   tilemix_paged_decode: one query token per sequence against its cached tokens; O and the
           log-sum-exp of the scores

``own`` chooses between the library's kernels and the same operators in elementary torch operations.
"""

import math
import random

import torch

own = False

TOP = {"int8": 127.0, "e4m3": 448.0}
FORMATS = {"fp16": torch.float16, "bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}


# ------------------------------------------------------------------------------------ cases

def listed():
    return [
        # One token of one short chat of a small multi-head model: launch latency.
        dict(name="append-token-mha-d64", kind="append", B=1, Hk=2, d=64, page=16, fmt="fp16", dtype="fp16",
             new_lo=1, new_hi=1, old_lo=999, old_hi=999),
        # The new tokens of a serving batch, one per sequence, between two decode steps.
        dict(name="append-step-b64-int8", kind="append", B=64, Hk=8, d=128, page=64, fmt="int8", dtype="fp16",
             new_lo=1, new_hi=1, old_lo=63, old_hi=8191),
        # A prompt of 8K tokens, cached after its prefill.
        dict(name="append-prompt-8k-int8", kind="append", B=1, Hk=8, d=128, page=64, fmt="int8", dtype="fp16",
             new_lo=8192, new_hi=8192, old_lo=0, old_hi=0),
        # The prompts of a packed batch, behind prefixes that are cached already; small pages.
        dict(name="append-packed-b24-e4m3", kind="append", B=24, Hk=8, d=128, page=16, fmt="e4m3", dtype="bf16",
             new_lo=5, new_hi=16000, old_lo=0, old_hi=1500),
        # The prefix of one chat, read back for the prefill of its next turn.
        dict(name="gather-chat-d64-bf16", kind="gather", B=1, Hk=2, d=64, page=32, fmt="bf16", dtype="bf16",
             lo=1000, hi=1000),
        # The prefixes of a packed batch, read back for a prefill in chunks.
        dict(name="gather-packed-b12-int8", kind="gather", B=12, Hk=8, d=128, page=64, fmt="int8", dtype="fp16",
             lo=333, hi=32768),
        # One decode step of one short chat: latency.
        dict(name="decode-1k-mha-d64-fp16", kind="decode", B=1, Hq=2, Hk=2, d=64, page=16, fmt="fp16", dtype="fp16",
             lo=1000, hi=1000, window=0),
        # A small serving batch with a cache in 16 bits.
        dict(name="decode-ragged-b8-bf16", kind="decode", B=8, Hq=32, Hk=8, d=128, page=32, fmt="bf16", dtype="bf16",
             lo=513, hi=8192, window=0),
        # A serving batch of chats of different lengths over an INT8 cache.
        dict(name="decode-ragged-b32-int8", kind="decode", B=32, Hq=32, Hk=8, d=128, page=64, fmt="int8", dtype="fp16",
             lo=64, hi=8192, window=0),
        # Four sequences of 64K tokens: memory bandwidth.
        dict(name="decode-64k-b4-int8", kind="decode", B=4, Hq=64, Hk=8, d=128, page=64, fmt="int8", dtype="fp16",
             lo=65536, hi=65536, window=0),
        # One document of 128K tokens, split over the whole GPU; small pages, E4M3.
        dict(name="decode-128k-e4m3", kind="decode", B=1, Hq=28, Hk=4, d=128, page=16, fmt="e4m3", dtype="bf16",
             lo=131072, hi=131072, window=0),
        # Sliding-window layers of a batch: the last 4096 tokens of longer caches.
        dict(name="decode-window-b16-int8", kind="decode", B=16, Hq=16, Hk=4, d=64, page=128, fmt="int8", dtype="bf16",
             lo=700, hi=20001, window=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# Most rows x channels of one operand: those of the four 64K sequences.
_MOST = 4 * 65536 * 8 * 128


def draw(rng):
    kind = rng.choice(["append", "gather", "decode", "decode"])
    Hq, Hk = rng.choice([(2, 2), (8, 8), (8, 2), (16, 4), (28, 4), (32, 8), (64, 8), (12, 4), (32, 1)])
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    fmt = rng.choice(["fp16", "bf16", "int8", "int8", "e4m3"])
    dtype = fmt if fmt in ("fp16", "bf16") else rng.choice(["fp16", "bf16"])
    B = _log_int(rng, 1, 96)
    case = dict(kind=kind, B=B, Hk=Hk, d=d, page=page, fmt=fmt, dtype=dtype)
    most = _MOST // (B * Hk * d)
    if fmt in ("fp16", "bf16"):
        most //= 2
    if kind == "append":
        old_hi = _log_int(rng, 1, min(most // 2, 16384))
        if rng.random() < 0.4:
            return dict(case, new_lo=1, new_hi=1, old_lo=rng.choice([0, old_hi]), old_hi=old_hi)
        hi = _log_int(rng, 2, min(most // 2, 65536))
        return dict(case, new_lo=_log_int(rng, 1, hi), new_hi=hi, old_lo=rng.choice([0, 0, old_hi]), old_hi=old_hi)
    hi = _log_int(rng, 1, min(most, 200000))
    case.update(lo=rng.choice([hi, _log_int(rng, 1, hi), 0]), hi=hi)
    if kind == "gather":
        return case
    window = 0 if rng.random() < 0.75 else _log_int(rng, 1, hi)
    return dict(case, Hq=Hq, window=window)


def _cdiv(a, b):
    return -(-a // b)


def _spread(n, lo, hi, turn):
    """n lengths of lo .. hi, spread over their logarithm, in an irregular order; the longest is hi."""
    if lo == hi:
        return [hi] * n
    u = [((i + turn) * 0.6180339887498949) % 1.0 for i in range(n)]
    got = [int(round(math.exp(math.log(lo + 1) + x * math.log((hi + 1) / (lo + 1))))) - 1 for x in u]
    got[u.index(max(u))] = hi
    return got


def _lengths(case):
    """(cached rows after the call, rows that the call writes or reads) of each sequence."""
    B = case["B"]
    if case["kind"] == "append":
        new = _spread(B, case["new_lo"], case["new_hi"], 0)
        return [o + x for o, x in zip(_spread(B, case["old_lo"], case["old_hi"], 7), new)], new
    lens = _spread(B, case["lo"], case["hi"], 0)
    return lens, [min(x, case["window"]) if case.get("window") else x for x in lens]


def work(case):
    lens, rows = _lengths(case)
    d, Hk = case["d"], case["Hk"]
    eight = case["fmt"] in TOP
    row = d + 4 if eight else 2 * d          # bytes of a cached row and its scale
    n = sum(rows) * Hk * 2                   # rows of K and V
    ids = 4 * (sum(_cdiv(x, case["page"]) for x in rows) + 2 * case["B"])
    if case["kind"] == "append":             # read the new rows, write the cache; 8 bits: read it, write the values
        return {"bytes": n * (2 * d + row + (row + 2 * d if eight else 0)) + ids, "flops": n * d * (3 if eight else 1)}
    if case["kind"] == "gather":
        return {"bytes": n * (row + 2 * d) + ids, "flops": n * d}
    heads = case["B"] * case["Hq"]
    return {"bytes": n * row + heads * (4 * d + 4) + ids, "flops": 4 * d * case["Hq"] * sum(rows)}


# ----------------------------------------------------------------------------------- inputs

def _quantise(x, fmt):
    """Codes and FP32 scales of rows x [.., d].  top * x is exact in FP32 and the quotient is rounded
    once, so that a code is the exactly rounded one."""
    top = TOP[fmt]
    x = x.float()
    a = x.abs().amax(-1, keepdim=True)
    q = torch.where(a > 0, x * top / a, torch.zeros_like(x))
    return (q.round() if fmt == "int8" else q).to(FORMATS[fmt]), (a / top).squeeze(-1)


def _pool(gen, shape, fmt, dtype, outliers):
    """Pages of N(0, 1) rows; with outliers, 1% of each head's channels (at least one) are 8 times larger."""
    P, H, page, d = shape
    X = torch.empty(shape, dtype=FORMATS[fmt], device="cuda")
    S = torch.empty(shape[:3], dtype=torch.float32, device="cuda") if fmt in TOP else None
    gain = torch.ones((H, 1, d), device="cuda")
    if outliers:
        ch = torch.rand((H, 1, d), generator=gen, device="cuda").argsort(-1)[..., : _cdiv(d, 100)]
        gain.scatter_(-1, ch, 8.0)
    step = max(1, (1 << 26) // (H * page * d))
    for at in range(0, P, step):
        x = torch.randn((min(step, P - at), H, page, d), generator=gen, device="cuda") * gain
        if fmt in TOP:
            X[at:at + step], S[at:at + step] = _quantise(x.to(FORMATS[dtype]), fmt)
        else:
            X[at:at + step] = x
    return X, S


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    lens, rows = _lengths(case)
    B, Hk, d, page, fmt = case["B"], case["Hk"], case["d"], case["page"], case["fmt"]
    dtype = FORMATS[case["dtype"]]
    per = max(1, _cdiv(max(lens), page))
    pages = B * per + 3                      # a pool has pages that nobody uses, too
    order = torch.randperm(pages, generator=gen, device="cuda")[: B * per]
    K, dK = _pool(gen, (pages, Hk, page, d), fmt, case["dtype"], True)
    V, dV = _pool(gen, (pages, Hk, page, d), fmt, case["dtype"], False)
    s = dict(kind=case["kind"], fmt=fmt, dtype=dtype, page=page, K=K, V=V, dK=dK, dV=dV,
             table=order.to(torch.int32).view(B, per).contiguous(),
             lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if case["kind"] == "decode":
        s.update(Q=torch.randn((B, 1, case["Hq"], d), generator=gen, device="cuda").to(dtype),
                 scale=1.0 / math.sqrt(d), window=case["window"])
        return s
    cu = [0]
    for x in rows:
        cu.append(cu[-1] + x)
    step = case["kind"] == "append" and case["new_lo"] == case["new_hi"] == 1
    s.update(cu=None if step else torch.tensor(cu, dtype=torch.int32, device="cuda"), most=max(rows), total=cu[-1])
    if case["kind"] == "append":
        shape = (B, 1, Hk, d) if step else (cu[-1], Hk, d)
        s["newK"], s["newV"] = (torch.randn(shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    return s


# -------------------------------------------------------------------------------------- run

def _slots(s):
    """(page, slot) of the rows that an append or gather deals with, in the order of the packed rows."""
    cu = s["cu"]
    if cu is None:
        cu = torch.arange(s["lens"].shape[0] + 1, dtype=torch.int32, device="cuda")
    t = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    at = (s["lens"][b] - cu[1:][b] + t).long()
    return s["table"][b, at // s["page"]].long(), at % s["page"]


def _read(X, scale, page, slot):
    x = X.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn) if X.dtype == torch.float8_e4m3fn else X[page, :, slot]
    return x.float() if scale is None else x.float() * scale[page, :, slot][..., None]


def _gather_plain(s):
    page, slot = _slots(s)
    shape = (s["lens"].shape[0], 1, *s["K"].shape[1::2]) if s["cu"] is None else (s["total"], *s["K"].shape[1::2])
    return tuple(_read(X, S, page, slot).to(s["dtype"]).view(shape) for X, S in ((s["K"], s["dK"]), (s["V"], s["dV"])))


def _write_plain(X, scale, x, fmt, page, slot):
    x = x.reshape(-1, *x.shape[-2:])
    if scale is None:
        X[page, :, slot] = x
        return
    q, r = _quantise(x, fmt)
    X.view(torch.uint8)[page, :, slot] = q.view(torch.uint8)
    scale[page, :, slot] = r


def _decode_plain(s):
    Q, table, page = s["Q"], s["table"], s["page"]
    B, _, Hq, d = Q.shape
    Hk, cap = s["K"].shape[1], table.shape[1] * page
    lens = s["lens"].long()[:, None]
    n = min(s["window"], cap) if s["window"] else cap
    at = (lens - s["window"]).clamp(min=0) * (s["window"] > 0) + torch.arange(n, device="cuda")
    seen = (at < lens)[:, None, None, :]
    at = at.clamp(max=cap - 1)
    ids, slot = table.gather(1, at // page).long(), at % page
    K = _read(s["K"], s["dK"], ids, slot).permute(0, 2, 3, 1)                       # [B, Hk, d, n]
    S = torch.matmul(Q.float().view(B, Hk, Hq // Hk, d), K.contiguous()) * s["scale"]
    del K
    S = torch.where(seen, S, torch.full_like(S, -math.inf))
    m = S.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    P = torch.exp(S - m)
    z = P.sum(-1, keepdim=True)
    V = _read(s["V"], s["dV"], ids, slot).permute(0, 2, 1, 3)                       # [B, Hk, n, d]
    O = torch.matmul(P, V.contiguous()) / torch.where(z > 0, z, torch.ones_like(z))
    return O.to(Q.dtype).view(B, 1, Hq, d), (m + torch.log(z)).view(B, Hq)


def run(state):
    s = state
    if own:
        import paper_2608_17336_amd as tm
        cache = tm.PagedCache(s["K"], s["V"], s["dK"], s["dV"])
        if s["kind"] == "decode":
            return tm.tilemix_paged_decode(cache, s["Q"], s["table"], s["lens"], s["scale"], window=s["window"],
                                           return_lse=True)
        if s["kind"] == "append":
            tm.tilemix_paged_append(cache, s["newK"], s["newV"], s["table"], s["lens"], s["cu"], s["most"])
            if s["fmt"] not in TOP:
                return s["K"], s["V"]
        return tm.tilemix_paged_gather(cache, s["table"], s["lens"], s["most"], s["cu"], s["total"], dtype=s["dtype"])
    if s["kind"] == "decode":
        return _decode_plain(s)
    if s["kind"] == "append":
        page, slot = _slots(s)
        _write_plain(s["K"], s["dK"], s["newK"], s["fmt"], page, slot)
        _write_plain(s["V"], s["dV"], s["newV"], s["fmt"], page, slot)
        if s["fmt"] not in TOP:
            return s["K"], s["V"]
    return _gather_plain(s)


# ------------------------------------------------------------------------------------ exact

def _values(x, fmt):
    """The values, in float64, that rows x have once they are held in ``fmt``: the nearest multiple of the
    row's step (int8), or the nearest number of four significant bits down to 2^-9 (e4m3), half to even."""
    x = x.double()
    if fmt not in TOP:
        return x
    a = x.abs().amax(-1, keepdim=True)
    unit = torch.where(a > 0, a, torch.ones_like(a)) / TOP[fmt]
    y = x / unit
    if fmt == "int8":
        return torch.round(y) * unit * (a > 0)
    step = torch.exp2(torch.frexp(y)[1].clamp(min=-5).double() - 4)
    return torch.round(y / step) * step * unit * (a > 0)


def exact(case, seed):
    s = prepare(case, seed)
    lens, rows = _lengths(case)
    page, fmt, Hk, d = case["page"], case["fmt"], case["Hk"], case["d"]
    table = s["table"].long()

    def cached(X, S, b, lo, hi):
        """Rows lo .. hi of sequence b in float64, [rows, Hk, d]."""
        ids = table[b].repeat_interleave(page)[lo:hi] * page + torch.arange(lo, hi, device="cuda") % page
        x = X.view(torch.int8) if X.dtype.itemsize == 1 else X.view(torch.int16)
        x = x.transpose(1, 2).reshape(-1, Hk, d)[ids].view(X.dtype).double()
        return x if S is None else x * S.transpose(1, 2).reshape(-1, Hk)[ids][..., None].double()

    if case["kind"] == "append":
        if fmt in TOP:
            return tuple(_values(s[k], fmt) for k in ("newK", "newV"))
        got = []
        for X, x in ((s["K"], s["newK"]), (s["V"], s["newV"])):
            out, x, at = X.double(), x.reshape(-1, Hk, d).double(), 0
            for b, (L, n) in enumerate(zip(lens, rows)):
                for t in range(L - n, L):
                    out[table[b, t // page], :, t % page] = x[at + t - (L - n)]
                at += n
            got.append(out)
        return tuple(got) if sum(rows) <= 20000 else None
    if case["kind"] == "gather":
        return tuple(torch.cat([cached(X, S, b, 0, L) for b, L in enumerate(lens)])
                     for X, S in ((s["K"], s["dK"]), (s["V"], s["dV"])))
    B, Hq = case["B"], case["Hq"]
    O = torch.zeros((B, 1, Hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    G = Hq // Hk
    for b, (L, n) in enumerate(zip(lens, rows)):
        for lo in range(L - n, L, 1 << 15):      # parts of the sequence, joined by their log-sum-exp
            hi = min(L, lo + (1 << 15))
            K, V = cached(s["K"], s["dK"], b, lo, hi), cached(s["V"], s["dV"], b, lo, hi)
            for h in range(Hq):
                sc = K[:, h // G] @ s["Q"][b, 0, h].double() * s["scale"]
                part = torch.logsumexp(sc, 0)
                both = torch.logaddexp(lse[b, h], part)
                o = torch.exp(sc - part) @ V[:, h // G]
                O[b, 0, h] = O[b, 0, h] * torch.exp(lse[b, h] - both) + o * torch.exp(part - both)
                lse[b, h] = both
    return O, lse


if __name__ == "__main__":
    for c in listed() + [draw(random.Random(i)) for i in range(6)]:
        print(c, work(c))
