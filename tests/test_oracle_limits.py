"""Pins of the oracles of drawing under limits and of the page calls: by hand, by enumeration, and by the rules a pool keeps."""
import numpy as np
import pytest

from oracle import decode_oracle as dec
from oracle import limits_oracle as lim
from oracle import pages_oracle as pg


def test_limits_by_hand():
    z = np.log([0.05, 0.4, 0.1, 0.25, 0.2])
    keep = lambda **kw: lim.kept(z, 1.0, **kw)[1].tolist()
    assert keep() == [1, 3, 4, 2, 0]
    assert keep(top_k=2) == [1, 3] and keep(top_k=9) == keep(top_k=-1) == keep()
    assert keep(top_p=0.39) == [1] and keep(top_p=0.41) == [1, 3] and keep(top_p=0.0) == [1] and keep(top_p=-2.0) == [1]
    assert keep(min_p=0.45) == [1, 3, 4] and keep(min_p=1.0) == keep(min_p=7.0) == [1] and keep(min_p=-1.0) == keep()
    # top-p is of what top-k leaves: 0.4 / 0.65 > 0.6
    assert keep(top_k=2, top_p=0.6) == [1] and keep(top_p=0.6) == [1, 3]
    token, logp, n, _ = lim.sample(z, 1.0, 0.3, top_k=2)
    assert (token, n) == (1, 2) and logp == pytest.approx(np.log(0.4 / 0.65))
    assert lim.sample(z, 1.0, 0.62, top_k=2)[0] == 3 and lim.sample(z, 0.0, 0.9)[:3] == (1, 0.0, 1)


def test_equal_tokens_stay_from_the_lowest_id_on():
    z = np.array([1.0, 2.0, 2.0, -np.inf, 2.0, 2.0])
    assert lim.kept(z, 1.0, top_k=3)[1].tolist() == [1, 2, 4]
    assert lim.kept(z, 0.001, top_p=0.5)[1].tolist() == [1, 2]
    assert lim.kept(z, 1.0)[1].tolist() == [1, 2, 4, 5, 0]
    assert lim.sample(np.full(4, -np.inf), 1.0, 0.5)[0] == -1 and lim.sample(np.array([0.0, np.nan]), 1.0, 0.5)[0] == -1


def test_draws_follow_the_limited_distribution():
    rng = np.random.default_rng(0)
    z = rng.normal(size=12) * 2
    w, ids, _ = lim.kept(z, 0.8, top_k=6, top_p=0.9, min_p=0.05)
    p = np.zeros(12)
    p[ids] = w[ids] / w[ids].sum()
    n = 20000
    counts = np.bincount([lim.sample(z, 0.8, (i + 0.5) / n, top_k=6, top_p=0.9, min_p=0.05)[0] for i in range(n)], minlength=12)
    assert np.abs(counts / n - p).max() <= 1.0 / n     # a regular grid of u: each token has its share, to one grid step


def test_verification_without_limits_is_the_plain_one_and_with_them_that_of_the_masked_row():
    rng = np.random.default_rng(1)
    for trial in range(60):
        g, V = 8, 24
        parent = np.array([rng.integers(-1, n) if n else -1 for n in range(g)])
        token, target = rng.integers(0, V, g), rng.normal(size=(1 + g, V)) * 2
        u, ub = rng.random(g), rng.random()
        args = (parent, token, np.arange(1, g + 1), target, 0.9, u, ub, g)
        assert lim.verify(*args)[:3] == dec.verify(*args)[:3]
        cut = np.full_like(target, -np.inf)
        for r in range(1 + g):
            ids = lim.kept(target[r], 0.9, top_k=7, top_p=0.8)[1]
            cut[r, ids] = target[r, ids]
        assert lim.verify(*args, top_k=7, top_p=0.8)[:3] == dec.verify(parent, token, np.arange(1, g + 1), cut, 0.9, u, ub, g)[:3]


def pool_of(S, width, n_pages):
    return dict(page_table=np.full((S, width), -1, np.int32), kv_len=np.zeros(S, np.int32), held=np.zeros(S, np.int32),
                ref_count=np.zeros(n_pages, np.int32))


def test_pages_by_hand():
    p, copies, bad, short = pg.resize(pool_of(3, 4, 10), [10, -1, 3], 4)
    assert not (copies or bad or short)
    assert p["page_table"].tolist() == [[0, 1, 2, -1], [-1] * 4, [3, -1, -1, -1]] and p["held"].tolist() == [3, 0, 1]
    p["kv_len"][:] = [6, 0, 3]
    q, bad = pg.fork(p, [2, 0, 2], 4)                 # 1 becomes what 0 was, 0 what 2 is
    assert not bad and q["page_table"].tolist() == [[3, -1, -1, -1], [0, 1, -1, -1], [3, -1, -1, -1]]
    assert q["kv_len"].tolist() == [3, 6, 3] and q["ref_count"].tolist() == [1, 1, 0, 2, 0, 0, 0, 0, 0, 0]
    r, copies, bad, short = pg.resize(q, [5, 8, 3], 4)  # 0 writes behind its 3 entries, 2 does not
    assert copies == [(3, 2, 3)] and r["page_table"].tolist() == [[2, 4, -1, -1], [0, 1, -1, -1], [3, -1, -1, -1]]
    assert r["ref_count"].tolist() == [1, 1, 1, 1, 1, 0, 0, 0, 0, 0]
    t, copies, bad, short = pg.resize(r, [16, 0, 16], 4)
    assert not short and t["held"].tolist() == [4, 0, 4] and t["page_table"][2].tolist() == [3, 7, 8, 9]
    assert t["page_table"][1].tolist() == [-1] * 4 and t["ref_count"].tolist() == [0, 0, 1, 1, 1, 1, 1, 1, 1, 1]
    u, copies, bad, short = pg.resize(r, [16, 16, 16], 4)   # five pages are free: 0 and 1 ask for two each, 2 for three
    assert short and u["held"].tolist() == [4, 4, 1]
    table, counts, used, moves = pg.compact(t)
    assert used == 8 and moves == [(8, 0), (9, 1)] and table[2].tolist() == [3, 7, 0, 1] and counts.tolist() == [1] * 8 + [0, 0]


def test_pools_keep_their_rules():
    rng = np.random.default_rng(2)
    page, S, width, n_pages = 4, 6, 8, 30
    p = pool_of(S, width, n_pages)
    for step in range(300):
        kind = rng.integers(3)
        if kind == 0:
            p, bad = pg.fork(p, rng.integers(-1, S, S), page)
        elif kind == 1:
            p, copies, bad, short = pg.resize(p, rng.integers(-1, width * page + 1, S), page)
            for s in range(S):                         # entries are written into what a sequence holds alone
                j = int(p["kv_len"][s]) // page
                while j < p["held"][s] and p["ref_count"][p["page_table"][s][j]] == 1 and p["kv_len"][s] < (j + 1) * page:
                    p["kv_len"][s] += rng.integers(0, (j + 1) * page - p["kv_len"][s] + 1)
                    break
        else:
            before = p
            table, counts, used, moves = pg.compact(p)
            p = dict(p, page_table=table, ref_count=counts)
            assert (counts[:used] > 0).all() and (counts[used:] == 0).all()
            where = dict(moves)
            assert all(table[s][j] == where.get(before["page_table"][s][j], before["page_table"][s][j]) for s in range(S) for j in range(width))
            bad = False
        assert not bad
        pg.check(p, page)
