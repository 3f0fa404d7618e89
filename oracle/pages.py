"""Oracle: pages for new tokens (test infrastructure only).

One sequence after the other, in plain Python, from the definition: a sequence of L tokens holds the page-table
entries first .. ceil(L / page) - 1; first is 0, and with a window moves to floor(max(L - window, 0) / page) when the
sequence grows.

Pins: tests/test_oracle_pages.py.
"""

from __future__ import annotations


def reserve(table, lens, wanted, page, ids, head, count, window=0, first=None, total=0):
    """table [B][max_pages], ids [N] (a ring) and the lists of lengths and first entries are copied.  Returns a dict of
    table, ids, head, count, refused, seqlens, first, cu_seqlens, positions and slots [total]."""
    first = list(first) if first else [0] * len(lens)
    table, ids = [list(row) for row in table], list(ids)
    N, per = len(ids), len(table[0])
    free = [ids[(head + i) % N] for i in range(count)]
    asked, given, refused, out, cu, rows = 0, [], 0, [], [0], []
    for b, (o, n) in enumerate(zip(lens, wanted)):
        o, n = min(max(o, 0), per * page), max(n, 0)
        low, have, new_have = first[b], -(-o // page), -(-n // page)
        new_low = max(low, max(n - window, 0) // page if window else 0)
        needs = list(range(max(have, new_low), new_have)) if n > o and n <= per * page else []
        asked += len(needs)
        if n > per * page or (needs and asked > count):
            refused += 1
            out.append(o)
            cu.append(cu[-1])
            continue
        if n > o:
            back = range(low, min(new_low, have))
            first[b] = new_low
        else:
            back = range(max(new_have, low), have)
            first[b] = min(low, new_have)
        old = list(table[b])
        for e in back:
            given.append(old[e])
            table[b][e] = -1
        for e in range(have, new_have):
            table[b][e] = free.pop(0) if e in needs else -1
        out.append(n)
        cu.append(cu[-1] + max(n - o, 0))
        for t in range(o, n):
            e = t // page
            id = table[b][e] if e >= new_low else -1
            rows.append((t, id * page + t % page if id >= 0 else -1))
    taken = count - len(free)
    for j, id in enumerate(given[:N - count]):
        ids[(head + count + j) % N] = id
    rows = (rows + [(-1, -1)] * total)[:total]
    return dict(table=table, ids=ids, head=(head + taken) % N, count=count - taken + min(len(given), N - count), refused=refused,
                seqlens=out, first=first, cu_seqlens=cu, positions=[p for p, _ in rows], slots=[s for _, s in rows])
