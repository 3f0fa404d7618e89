"""Timed cases of what a server does around a decode step: pages for new tokens, rotary positions, and a paged
key/value cache held in 4 bits.

  reserve  tilemix_paged_reserve: from the lengths that the sequences have and those that they want, pages are
           taken from and given back to a list of free ones; page table, lengths, the positions and slots of the
           new tokens
  rotary   tilemix_rotary: Q and K turned by their tokens' positions, or, inverse, the gradient of that
  append   tilemix_paged_append into an MXFP4 pool, read back by tilemix_paged_gather, so that the outputs
           are the values that the codes stand for
  gather   tilemix_paged_gather: the rows of every sequence, packed and in 16 bits
  decode   tilemix_paged_decode: one query token per sequence against its cached tokens; O and the log-sum-exp

An MXFP4 pool holds a row (a token's d channels of one head) as d / 2 bytes of E2M1 codes, the even channel in
the low four bits, and an exponent byte for each 32 channels: 2^(byte - 127).

``own`` chooses between the library's kernels and the same operators in elementary torch operations.
"""

import math
import random

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------ cases

def listed():
    return [
        # The next token of 64 chats: latency.
        dict(name="reserve-step-b64", kind="reserve", B=64, page=64, old_lo=63, old_hi=8191, new_lo=1, new_hi=1,
             done=0, short=False),
        # A busy server admits and finishes requests: every seventh is done, the others bring prompts or
        # parts of them, and not all get their pages.
        dict(name="reserve-admit-b256", kind="reserve", B=256, page=16, old_lo=0, old_hi=8000, new_lo=1, new_hi=16000,
             done=7, short=True),
        # One token of one short chat of a small multi-head model: latency.
        dict(name="rotary-token-mha-d64", kind="rotary", B=1, Hq=2, Hk=2, d=64, r=64, dtype="fp16", layout="half",
             new_lo=1, new_hi=1, old_lo=999, old_hi=999, slices=False, lengths=False, inverse=False, factor=1.0),
        # A prompt of 8K tokens, out of the slices of a fused projection.
        dict(name="rotary-prompt-8k", kind="rotary", B=1, Hq=32, Hk=8, d=128, r=128, dtype="fp16", layout="half",
             new_lo=8192, new_hi=8192, old_lo=0, old_hi=0, slices=True, lengths=False, inverse=False, factor=1.0),
        # The gradient of a packed batch whose positions are scaled for long contexts; half of each head turns.
        dict(name="rotary-grad-packed-b24", kind="rotary", B=24, Hq=28, Hk=4, d=128, r=64, dtype="bf16",
             layout="interleaved", new_lo=5, new_hi=16000, old_lo=0, old_hi=120000, slices=False, lengths=True,
             inverse=True, factor=8.0),
        # The new tokens of a serving batch, one per sequence, between two decode steps.
        dict(name="append-step-b64", kind="append", B=64, Hk=8, d=128, page=64, dtype="fp16",
             new_lo=1, new_hi=1, old_lo=63, old_hi=8191),
        # The prompts of a packed batch, behind prefixes that are cached already; small pages.
        dict(name="append-packed-b24", kind="append", B=24, Hk=8, d=128, page=16, dtype="bf16",
             new_lo=5, new_hi=16000, old_lo=0, old_hi=1500),
        # The prefix of one chat, read back for the prefill of its next turn.
        dict(name="gather-chat-d64", kind="gather", B=1, Hk=2, d=64, page=32, dtype="bf16", lo=1000, hi=1000),
        # The prefixes of a packed batch, read back for a prefill in chunks.
        dict(name="gather-packed-b12", kind="gather", B=12, Hk=8, d=128, page=64, dtype="fp16", lo=333, hi=32768),
        # One decode step of one short chat: latency.
        dict(name="decode-1k-mha-d64", kind="decode", B=1, Hq=2, Hk=2, d=64, page=16, dtype="bf16",
             lo=1000, hi=1000, window=0),
        # A serving batch of chats of different lengths.
        dict(name="decode-ragged-b32", kind="decode", B=32, Hq=32, Hk=8, d=128, page=64, dtype="fp16",
             lo=64, hi=8192, window=0),
        # Eight sequences of 64K tokens: memory bandwidth.
        dict(name="decode-64k-b8", kind="decode", B=8, Hq=64, Hk=8, d=128, page=64, dtype="fp16",
             lo=65536, hi=65536, window=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# Most rows x channels of one operand of the cache: those of the eight 64K sequences; of Q and K together: those
# of the packed gradient; most new tokens, and page-table entries.
_MOST, _MOST_TURNED, _MOST_TOKENS, _MOST_ENTRIES = 8 * 65536 * 8 * 128, 1 << 27, 1 << 19, 1 << 20


def draw(rng):
    kind = rng.choice(["reserve", "rotary", "rotary", "append", "gather", "decode", "decode", "decode"])
    Hq, Hk = rng.choice([(2, 2), (8, 8), (8, 2), (16, 4), (28, 4), (32, 8), (64, 8), (12, 4), (32, 1)])
    d = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    dtype = rng.choice(["fp16", "bf16"])
    if kind == "reserve":
        B = _log_int(rng, 1, 4096)
        hi = _log_int(rng, 1, max(1, min(32768, _MOST_TOKENS // B)))
        old = _log_int(rng, 1, max(1, min(65536, _MOST_ENTRIES // B * page - hi)))
        one = rng.random() < 0.4
        return dict(kind=kind, B=B, page=page, old_lo=rng.choice([0, old]), old_hi=old, new_lo=1, new_hi=1 if one else hi,
                    done=rng.choice([0, 0, 3, 11]), short=rng.random() < 0.3)
    B = _log_int(rng, 1, 96)
    if kind == "rotary":
        most = max(1, _MOST_TURNED // (B * (Hq + 2 * Hk) * d))
        hi = 1 if rng.random() < 0.3 else _log_int(rng, 1, min(most, 65536))
        old = _log_int(rng, 1, 1 << 20)
        return dict(kind=kind, B=B, Hq=Hq, Hk=Hk, d=d, r=rng.choice([d, d, d // 2, d // 4, 2 * rng.randrange(1, d // 2)]),
                    dtype=dtype, layout=rng.choice(["half", "interleaved"]), new_lo=rng.choice([hi, _log_int(rng, 1, hi)]),
                    new_hi=hi, old_lo=rng.choice([0, old]), old_hi=old, slices=rng.random() < 0.5,
                    lengths=rng.random() < 0.5, inverse=rng.random() < 0.3, factor=rng.choice([1.0, 4.0, 32.0]))
    case = dict(kind=kind, B=B, Hk=Hk, d=d, page=page, dtype=dtype)
    most = _MOST // (B * Hk * d)
    if kind == "append":
        most = min(most, _MOST_TOKENS * 8 // (B * Hk))
        old_hi = _log_int(rng, 1, max(1, min(most // 2, 16384)))
        if rng.random() < 0.4:
            return dict(case, new_lo=1, new_hi=1, old_lo=rng.choice([0, old_hi]), old_hi=old_hi)
        hi = _log_int(rng, 2, max(2, min(most // 2, 65536)))
        return dict(case, new_lo=_log_int(rng, 1, hi), new_hi=hi, old_lo=rng.choice([0, 0, old_hi]), old_hi=old_hi)
    if kind == "gather":
        most = min(most, _MOST_TOKENS * 8 // (B * Hk))
    hi = _log_int(rng, 1, min(most, 200000))
    case.update(lo=rng.choice([hi, _log_int(rng, 1, hi), 0]), hi=hi)
    if kind == "gather":
        return case
    return dict(case, Hq=Hq, window=0 if rng.random() < 0.75 else _log_int(rng, 1, hi))


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
    """(tokens after the call, tokens that the call adds, turns or reads) of each sequence; of a reservation
    (tokens before, tokens wanted)."""
    B = case["B"]
    if case["kind"] in ("gather", "decode"):
        lens = _spread(B, case["lo"], case["hi"], 0)
        return lens, [min(x, case["window"]) if case.get("window") else x for x in lens]
    new = _spread(B, case["new_lo"], case["new_hi"], 0)
    old = _spread(B, case["old_lo"], case["old_hi"], 7)
    if case["kind"] == "reserve":
        return old, [0 if case["done"] and b % case["done"] == 2 else o + x for b, (o, x) in enumerate(zip(old, new))]
    return [o + x for o, x in zip(old, new)], new


def _reservation(case):
    """(new tokens, pages taken, pages given back) if every sequence is served."""
    old, want = _lengths(case)
    pages = [_cdiv(n, case["page"]) - _cdiv(o, case["page"]) for o, n in zip(old, want)]
    return sum(max(n - o, 0) for o, n in zip(old, want)), sum(max(x, 0) for x in pages), sum(max(-x, 0) for x in pages)


def work(case):
    if case["kind"] == "reserve":
        tokens, taken, given = _reservation(case)
        # Old and wanted lengths, new lengths, prefix sums; an id of each page read and written; position and slot.
        return {"bytes": 16 * case["B"] + 8 * (taken + given) + 12 * tokens, "flops": 2 * case["B"] + 4 * tokens}
    lens, rows = _lengths(case)
    d, Hk = case["d"], case["Hk"]
    if case["kind"] == "rotary":
        heads = sum(rows) * (case["Hq"] + Hk)
        return {"bytes": heads * 4 * d + (8 * case["B"] if case["lengths"] else 4 * sum(rows)) + 4 * case["r"],
                "flops": heads * 3 * case["r"] + sum(rows) * case["r"]}
    row = d // 2 + d // 32                   # bytes of a cached row and its exponents
    n = sum(rows) * Hk * 2                   # rows of K and V
    ids = 4 * (sum(_cdiv(x, case["page"]) for x in rows) + 2 * case["B"])
    if case["kind"] == "append":             # read the new rows, write the cache; read it, write the values
        return {"bytes": n * (2 * d + row + row + 2 * d) + ids, "flops": n * d * 3}
    if case["kind"] == "gather":
        return {"bytes": n * (row + 2 * d) + ids, "flops": n * d}
    heads = case["B"] * case["Hq"]
    return {"bytes": n * row + heads * (4 * d + 4) + ids, "flops": 4 * d * case["Hq"] * sum(rows)}


# ----------------------------------------------------------------------------------- inputs

def _quantise(x):
    """E2M1 codes [.., d / 2] (bytes) and exponent bytes [.., d / 32] of rows x [.., d] of 16-bit values.  The exponent
    of a block is the least one, from -127 on, with all magnitudes below 7 2^e; x 2^-e is exact in FP32."""
    x = x.float().unflatten(-1, (-1, 32))
    f, k = torch.frexp(x.abs().amax(-1))
    e = (k - 3 + (f >= 0.875).int()).clamp(min=-127)
    e = torch.where(f > 0, e, torch.full_like(e, -127))
    h = e // 2                               # in two steps: 2^127 and 2^-127 are no FP32 numbers to rely on
    y = torch.ldexp(torch.ldexp(x, -h[..., None]), (h - e)[..., None])
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * torch.signbit(y)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _pool(gen, shape, outliers):
    """Pages of N(0, 1) rows; with outliers, 1% of each head's channels (at least one) are 8 times larger."""
    P, H, page, d = shape
    X = torch.empty((P, H, page, d // 2), dtype=torch.uint8, device="cuda")
    S = torch.empty((P, H, page, d // 32), dtype=torch.uint8, device="cuda")
    gain = torch.ones((H, 1, d), device="cuda")
    if outliers:
        ch = torch.rand((H, 1, d), generator=gen, device="cuda").argsort(-1)[..., : _cdiv(d, 100)]
        gain.scatter_(-1, ch, 8.0)
    step = max(1, (1 << 26) // (H * page * d))
    for at in range(0, P, step):
        x = torch.randn((min(step, P - at), H, page, d), generator=gen, device="cuda") * gain
        X[at:at + step], S[at:at + step] = _quantise(x.half())
    return X, S


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _prefix(x):
    cu = [0]
    for n in x:
        cu.append(cu[-1] + n)
    return cu


def _prepare_reserve(case, gen):
    old, want = _lengths(case)
    B, page = case["B"], case["page"]
    tokens, taken, given = _reservation(case)
    have = [_cdiv(x, page) for x in old]
    per = max(1, *(_cdiv(x, page) for x in old + want))
    held = sum(have)
    count = taken // 2 if case["short"] else taken + B
    P = held + count + 3                     # (a few pages are in other hands)
    order = torch.randperm(P, generator=gen, device="cuda").int()
    table = torch.full((B, per), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(per, device="cuda") < _ints(have)[:, None]] = order[:held]
    room = P + 5
    ids = torch.full((room,), -1, dtype=torch.int32, device="cuda")
    head = room // 2
    ids[(head + torch.arange(count, device="cuda")) % room] = order[held:held + count]
    return dict(kind="reserve", page=page, table=table, lens=_ints(old), want=_ints(want), ids=ids,
                free=_ints([head, count, 0, 0]), total=tokens + 17,   # rows of padding, as for a captured graph
                new_free=torch.empty(4, dtype=torch.int32, device="cuda"),
                new_lens=torch.empty(B, dtype=torch.int32, device="cuda"))


def _prepare_rotary(case, gen):
    lens, rows = _lengths(case)
    Hq, Hk, d, r = case["Hq"], case["Hk"], case["d"], case["r"]
    total, dtype = sum(rows), TYPES[case["dtype"]]
    heads = (Hq, Hk, Hk) if case["slices"] else (Hq, Hk)
    if case["slices"]:
        X = torch.randn((total, sum(heads), d), generator=gen, device="cuda").to(dtype)
        Q, K = X[:, :Hq], X[:, Hq:Hq + Hk]
    else:
        Q, K = (torch.randn((total, h, d), generator=gen, device="cuda").to(dtype) for h in heads)
    freq = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r) / case["factor"]
    cu = _ints(_prefix(rows))
    at = torch.arange(total, dtype=torch.int32, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), at, right=True)
    pos = (_ints(lens)[b] - cu[1:][b] + at).int()
    return dict(kind="rotary", Q=Q, K=K, freq=freq, pos=None if case["lengths"] else pos, lens=_ints(lens), cu=cu,
                most=max(rows), layout=case["layout"], inverse=case["inverse"], r=r,
                gain=1.0 if case["factor"] == 1.0 else 0.1 * math.log(case["factor"]) + 1.0)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 29)
    if case["kind"] == "reserve":
        return _prepare_reserve(case, gen)
    if case["kind"] == "rotary":
        return _prepare_rotary(case, gen)
    lens, rows = _lengths(case)
    B, Hk, d, page = case["B"], case["Hk"], case["d"], case["page"]
    dtype = TYPES[case["dtype"]]
    per = max(1, _cdiv(max(lens), page))
    pages = B * per + 3                      # a pool has pages that nobody uses, too
    order = torch.randperm(pages, generator=gen, device="cuda")[: B * per]
    (K, dK), (V, dV) = (_pool(gen, (pages, Hk, page, d), outliers) for outliers in (True, False))
    s = dict(kind=case["kind"], dtype=dtype, page=page, K=K.view(torch.float4_e2m1fn_x2), V=V.view(torch.float4_e2m1fn_x2),
             dK=dK.view(torch.float8_e8m0fnu), dV=dV.view(torch.float8_e8m0fnu),
             table=order.to(torch.int32).view(B, per).contiguous(), lens=_ints(lens))
    if case["kind"] == "decode":
        s.update(Q=torch.randn((B, 1, case["Hq"], d), generator=gen, device="cuda").to(dtype),
                 scale=1.0 / math.sqrt(d), window=case["window"])
        return s
    step = case["kind"] == "append" and case["new_lo"] == case["new_hi"] == 1
    s.update(cu=None if step else _ints(_prefix(rows)), most=max(rows), total=sum(rows))
    if case["kind"] == "append":
        shape = (B, 1, Hk, d) if step else (sum(rows), Hk, d)
        s["newK"], s["newV"] = (torch.randn(shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    return s


# -------------------------------------------------------------------------------------- run

def _reserve_plain(s):
    page, table, ids, total = s["page"], s["table"], s["ids"], s["total"]
    per, N = table.shape[1], ids.shape[0]
    o, n = s["lens"].long(), s["want"].long()
    head, count = s["free"][0].long(), s["free"][1].long()
    have, want = (o + page - 1) // page, (n + page - 1) // page
    fits = n <= per * page
    need = torch.where(fits, (want - have).clamp(min=0), torch.zeros_like(n))
    ok = fits & ((need == 0) | (need.cumsum(0) <= count))
    take = torch.where(ok, need, torch.zeros_like(n))
    give = (have - want).clamp(min=0)
    lens = torch.where(ok, n, o)
    e = torch.arange(per, device="cuda")
    taken = (e >= have[:, None]) & (e < (have + take)[:, None])
    given = (e >= (have - give)[:, None]) & (e < have[:, None])
    start = head + take.cumsum(0) - take - have
    to = head + count + give.cumsum(0) - give - want
    place = torch.where(given, (to[:, None] + e) % N, torch.full_like(given, N, dtype=torch.long))
    ring = torch.cat([ids, ids[:1]]).scatter(0, place.flatten(), table.flatten())[:N]   # (the last is what is not given)
    new = torch.where(taken, ids[(start[:, None] + e) % N], table)
    new = torch.where(given, torch.full_like(new, -1), new)
    table.copy_(new)
    ids.copy_(ring)
    rows = (lens - o).clamp(min=0)
    cu = torch.cat([rows.new_zeros(1), rows.cumsum(0)])
    i = torch.arange(total, device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), i, right=True).clamp(max=o.shape[0] - 1)
    some = i < cu[-1]
    pos = o[b] + i - cu[b]
    slot = table[b, (pos // page).clamp(max=per - 1)].long() * page + pos % page
    none = torch.full_like(pos, -1)
    free = torch.stack([(head + take.sum()) % N, count + give.sum() - take.sum(), (~ok).sum()])
    return (table, ids, free.int(), lens.int(), cu.int(), torch.where(some, pos, none).int(), torch.where(some, slot, none))


def _rotary_plain(s):
    r, pos = s["r"], s["pos"]
    if pos is None:
        at = torch.arange(s["Q"].shape[0], device="cuda")
        b = torch.searchsorted(s["cu"][1:].contiguous(), at, right=True)
        pos = s["lens"][b] - s["cu"][1:][b] + at
    angle = pos.double()[:, None] * s["freq"]
    c, z = (torch.cos(angle) * s["gain"]).float()[:, None], (torch.sin(angle) * s["gain"]).float()[:, None]
    if s["inverse"]:
        z = -z

    def turn(X):
        x = X.float()
        if s["layout"] == "half":
            x1, x2 = x[..., : r // 2], x[..., r // 2:r]
            y = torch.cat([x1 * c - x2 * z, x2 * c + x1 * z], -1)
        else:
            x1, x2 = x[..., 0:r:2], x[..., 1:r:2]
            y = torch.stack([x1 * c - x2 * z, x2 * c + x1 * z], -1).flatten(-2)
        return torch.cat([y, x[..., r:]], -1).to(X.dtype)

    return turn(s["Q"]), turn(s["K"])


def _slots(s):
    """(page, slot) of the rows that an append or gather deals with, in the order of the packed rows."""
    cu = s["cu"]
    if cu is None:
        cu = torch.arange(s["lens"].shape[0] + 1, dtype=torch.int32, device="cuda")
    t = torch.arange(s["total"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    at = (s["lens"][b] - cu[1:][b] + t).long()
    return s["table"][b, at // s["page"]].long(), at % s["page"]


def _read(X, S, page, slot):
    """Rows in FP32, [.., d]."""
    code = X.view(torch.uint8)[page, :, slot].int()
    value = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
    x = torch.stack([value[code & 15], value[code >> 4]], -1).flatten(-2)
    del code
    e = S.view(torch.uint8)[page, :, slot].int() - 127
    unit = torch.ldexp(torch.ldexp(torch.ones_like(e, dtype=torch.float32), e // 2), e - e // 2)
    return (x.unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def _gather_plain(s):
    page, slot = _slots(s)
    Hk, d = s["K"].shape[1], 2 * s["K"].shape[3]
    shape = (s["lens"].shape[0], 1, Hk, d) if s["cu"] is None else (s["total"], Hk, d)
    return tuple(_read(X, S, page, slot).to(s["dtype"]).view(shape) for X, S in ((s["K"], s["dK"]), (s["V"], s["dV"])))


def _append_plain(s):
    page, slot = _slots(s)
    for X, S, x in ((s["K"], s["dK"], s["newK"]), (s["V"], s["dV"], s["newV"])):
        X.view(torch.uint8)[page, :, slot], S.view(torch.uint8)[page, :, slot] = _quantise(x.reshape(-1, *x.shape[-2:]))


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
    if not own:
        if s["kind"] == "append":
            _append_plain(s)
        return {"reserve": _reserve_plain, "rotary": _rotary_plain, "append": _gather_plain, "gather": _gather_plain,
                "decode": _decode_plain}[s["kind"]](s)
    import paper_2608_17336_amd as tm
    if s["kind"] == "reserve":
        got = tm.tilemix_paged_reserve(tm.PageList(s["ids"], s["free"]), s["table"], s["lens"], s["want"], s["page"],
                                       total=s["total"], state_out=s["new_free"], seqlens_out=s["new_lens"])
        return s["table"], s["ids"], s["new_free"][:3], got.seqlens, got.cu_seqlens, got.positions, got.slots
    if s["kind"] == "rotary":
        at = dict(positions=s["pos"]) if s["pos"] is not None else dict(seqlens_k=s["lens"], cu_seqlens=s["cu"])
        return tm.tilemix_rotary(s["Q"], s["K"], s["freq"], **at, layout=s["layout"], magnitude=s["gain"],
                                 inverse=s["inverse"])
    cache = tm.PagedCache(s["K"], s["V"], s["dK"], s["dV"])
    if s["kind"] == "decode":
        return tm.tilemix_paged_decode(cache, s["Q"], s["table"], s["lens"], s["scale"], window=s["window"],
                                       return_lse=True)
    if s["kind"] == "append":
        tm.tilemix_paged_append(cache, s["newK"], s["newV"], s["table"], s["lens"], s["cu"], s["most"])
    return tm.tilemix_paged_gather(cache, s["table"], s["lens"], s["most"], s["cu"], s["total"], dtype=s["dtype"])


# ------------------------------------------------------------------------------------ exact

def _values(x):
    """The values, in float64, that rows x have once they are held in MXFP4: of each 32 channels the nearest
    multiples, half to even, of a step that is 2^(e - 1) up to 2^(e + 1) and doubles with each power of two beyond."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -127.0)
    some = top > 0
    e = torch.where(some, torch.floor(torch.log2(torch.where(some, top, torch.ones_like(top)))) - 2, e)
    e = torch.where(top >= 7 * torch.exp2(e), e + 1, e).clamp(min=-127.0)
    unit = torch.exp2(e)
    y = y / unit
    step = 0.5 * torch.exp2((torch.frexp(y)[1] - 1).clamp(min=0).double())
    return (torch.round(y / step) * step * unit).flatten(-2)


def _exact_rotary(s):
    """As products of complex numbers."""
    pos, r = s["pos"], s["r"]
    if pos is None:
        cu = s["cu"].tolist()
        pos = torch.cat([torch.arange(n - (hi - lo), n, device="cuda") for n, lo, hi in zip(s["lens"].tolist(), cu, cu[1:])])
    angle = pos.double()[:, None, None] * s["freq"] * (-1.0 if s["inverse"] else 1.0)
    w = torch.polar(torch.full_like(angle, s["gain"]), angle)
    out = []
    for X in (s["Q"], s["K"]):
        y = X.double()
        pairs = torch.arange(r, device="cuda").view(2, -1) if s["layout"] == "half" else torch.arange(r, device="cuda").view(-1, 2).T
        x = torch.complex(y[..., pairs[0]], y[..., pairs[1]]) * w
        y[..., pairs[0]], y[..., pairs[1]] = x.real, x.imag
        out.append(y)
    return tuple(out)


def exact(case, seed):
    if case["kind"] == "reserve":
        return None                          # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    if case["kind"] == "append":
        return _values(s["newK"]), _values(s["newV"])
    lens, rows = _lengths(case)
    page, Hk, d = case["page"], case["Hk"], case["d"]
    table = s["table"].long()
    value = torch.tensor(E2M1, dtype=torch.float64, device="cuda")

    def cached(X, S, b, lo, hi):
        """Rows lo .. hi of sequence b in float64, [rows, Hk, d]."""
        ids = table[b].repeat_interleave(page)[lo:hi] * page + torch.arange(lo, hi, device="cuda") % page
        code = X.view(torch.uint8).transpose(1, 2).reshape(-1, Hk, d // 2)[ids].long()
        code = torch.stack([code % 16, code // 16], -1).view(hi - lo, Hk, d)
        x = value[code % 8] * (1 - 2 * (code // 8))
        e = S.view(torch.uint8).transpose(1, 2).reshape(-1, Hk, d // 32)[ids].double() - 127
        return x * torch.exp2(e).repeat_interleave(32, -1)

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
