"""Oracle of the page calls: one sequence and one page at a time, on the host.

A pool is a dict of numpy int arrays page_table [S, max_pages], kv_len [S], held [S], ref_count [n_pages]; a cache is an
array [n_layers, n_pages, page_size, ...].  The functions return new pools; `copies` lists (from, to, entries).  A sequence
whose numbers do not allow the call stays as it is; what is given back need not be sound (a name that is no page is
reported, and skipped)."""
from __future__ import annotations

import numpy as np


def copy_of(pool):
    return {k: np.array(v) for k, v in pool.items()}


def fits(pool, s, page):
    held, n = int(pool["held"][s]), int(pool["kv_len"][s])
    return 0 <= held <= pool["page_table"].shape[1] and 0 <= n <= held * page


def is_page(pool, p):
    return 0 <= p < len(pool["ref_count"])


def fork(pool, parent, page):
    """(pool, bad)."""
    out, bad = copy_of(pool), False
    S, width = pool["page_table"].shape
    for s in range(S):
        f = int(parent[s])
        if f == s:
            continue
        if not -1 <= f < S or not 0 <= pool["held"][s] <= width or (f >= 0 and not fits(pool, f, page)):
            bad = True
            continue
        n = 0 if f < 0 else int(pool["kv_len"][f])
        pages = [int(p) for p in pool["page_table"][f][:-(-n // page)]] if f >= 0 else []
        if not all(is_page(pool, p) for p in pages):
            bad = True
            continue
        for p in pool["page_table"][s][:pool["held"][s]]:
            if is_page(pool, p):
                out["ref_count"][p] -= 1
            else:
                bad = True
        for p in pages:
            out["ref_count"][p] += 1
        out["page_table"][s] = pages + [-1] * (width - len(pages))
        out["kv_len"][s], out["held"][s] = n, len(pages)
    return out, bad


def resize(pool, want, page):
    """(pool, copies, bad, short)."""
    out, copies, bad, short = copy_of(pool), [], False, False
    S, width = pool["page_table"].shape
    free = [p for p in range(len(pool["ref_count"])) if pool["ref_count"][p] == 0]
    asked = 0                                    # by those before, whether they got it or not
    for s in range(S):
        w = int(want[s])
        if w < 0:
            continue
        if not fits(pool, s, page) or w > width * page:
            bad = True
            continue
        held, keep, need = int(pool["held"][s]), min(int(pool["kv_len"][s]), w), -(-w // page)
        row = [int(p) for p in pool["page_table"][s]]
        written = range(keep // page, min(held, need)) if w > keep else []
        if not all(is_page(pool, row[j]) for j in written):
            bad = True
            continue
        swaps = [j for j in written if pool["ref_count"][row[j]] > 1]
        slots = swaps + list(range(held, need))
        at, asked = asked, asked + len(slots)
        if slots and asked > len(free):
            short = True
            continue
        for j in range(need, held):
            if is_page(pool, row[j]):
                out["ref_count"][row[j]] -= 1
            else:
                bad = True
            out["page_table"][s][j] = -1
        for i, j in enumerate(slots):
            new = free[at + i]
            if j in swaps:
                out["ref_count"][row[j]] -= 1
                if j == keep // page and keep % page:
                    copies.append((row[j], new, keep % page))
            out["ref_count"][new] = 1
            out["page_table"][s][j] = new
        out["held"][s], out["kv_len"][s] = need, keep
    return out, copies, bad, short


def compact(pool):
    """(table, counts, pages in use, copies of whole pages as (from, to))."""
    ref = pool["ref_count"]
    n_used = int((ref > 0).sum())
    moves = list(zip([p for p in range(n_used, len(ref)) if ref[p] > 0], [p for p in range(n_used) if ref[p] <= 0]))
    where = dict(moves)
    table = np.array([[where.get(int(p), int(p)) for p in row] for row in pool["page_table"]], np.int32).reshape(pool["page_table"].shape)
    counts = np.where(ref > 0, ref, 0)
    for a, b in moves:
        counts[b], counts[a] = ref[a], 0
    return table, counts, n_used, moves


def check(pool, page):
    """The rules every pool keeps: counts are the names in held slots, and nothing is named behind them."""
    S, width = pool["page_table"].shape
    count = np.zeros(len(pool["ref_count"]), np.int64)
    for s in range(S):
        assert fits(pool, s, page)
        for j, p in enumerate(pool["page_table"][s]):
            if j < pool["held"][s]:
                count[p] += 1
            else:
                assert p == -1
    assert np.array_equal(count, pool["ref_count"])
