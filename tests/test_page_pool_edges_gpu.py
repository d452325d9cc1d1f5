"""The page calls where their documentation ends: pools without sequences, broken names, contexts without pages."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


def make(gto, S=4, n_pages=12, max_pages=5, page=4, layers=2):
    cfg = gto.make_decode_config(S=S, T=S, n_q_heads=1, n_kv_heads=1, head_dim=16, page_size=page, n_pages=n_pages, max_pages=max_pages,
                                 dtype="f32", flags=gto.GTO_DECODE_PAGES)
    k, v = (torch.randn((layers, n_pages, page, 1, 16), device=DEV) for _ in range(2))
    return gto.gto_decode_create(cfg, 0), cfg, k, v


@pytest.mark.parametrize("counts", [[0] * 12, [0, 2, 0, 0, 1, 0, 0, 1, 0, 0, 0, 3]])
def test_compact_of_a_pool_without_sequences(gto, counts):
    """The counts alone decide (whoever holds the pages); every output is written."""
    ctx, cfg, k, v = make(gto)
    pool = gto.alloc_page_pool(cfg, DEV, 0)
    pool["ref_count"].copy_(torch.tensor(counts))
    table, ref, used = torch.full((0, 5), -9, **I32), torch.full((12,), -9, **I32), torch.full((1,), -9, **I32)
    was = k.clone(), v.clone()
    gto.gto_pages_compact(ctx, pool, k, v, table, ref, used)
    assert gto.gto_decode_status(ctx) == 0
    n = sum(c > 0 for c in counts)
    assert used.item() == n
    moves = list(zip([p for p in range(n, 12) if counts[p]], [p for p in range(n) if not counts[p]]))
    want = [counts[p] if p < n else 0 for p in range(12)]
    for x, y in zip((k, v), was):
        for a, b in moves:
            y[:, b] = y[:, a]
            want[b] = counts[a]
        assert torch.equal(x, y)
    assert ref.tolist() == want and pool["ref_count"].tolist() == counts


def test_compact_of_a_pool_without_sequences_refuses_what_it_would_write_over(gto):
    ctx, cfg, k, v = make(gto)
    pool = gto.alloc_page_pool(cfg, DEV, 0)
    table, ref, used = torch.zeros((0, 5), **I32), torch.zeros(12, **I32), torch.zeros(1, **I32)
    for bad in (dict(ref=pool["ref_count"]), dict(used=pool["ref_count"][:1]), dict(used=ref[3:4])):
        args = dict(ref=ref, used=used) | bad
        with pytest.raises(gto.GtoError) as e:
            gto.gto_pages_compact(ctx, pool, k, v, table, args["ref"], args["used"])
        assert e.value.code == 1
    inside = torch.zeros((3, 5), **I32)
    gto.gto_pages_compact(ctx, pool, k, v, inside[1:1], ref, used)  # nothing lies over anything
    assert gto.gto_decode_status(ctx) == 0


# A page size of 4, 12 pages: sequence 0 holds pages 0 1 2 (9 entries), 1 holds 3 4 (5 entries), 2 and 3 nothing.
TABLE, LEN, HELD = [[0, 1, 2, -1, -1], [3, 4, -1, -1, -1], [-1] * 5, [-1] * 5], [9, 5, 0, 0], [3, 2, 0, 0]
COUNT = [1, 1, 1, 1, 1, 0, 0, 0, 0, 0, 0, 0]


def broken(gto, cfg, **at):
    pool = gto.alloc_page_pool(cfg, DEV)
    for n, x in (("page_table", TABLE), ("kv_len", LEN), ("held", HELD), ("ref_count", COUNT)):
        pool[n].copy_(torch.tensor(x))
    for n, (where, value) in at.items():
        pool[n][where] = value
    return pool


def numbers(pool):
    return {n: x.tolist() for n, x in pool.items()}


@pytest.mark.parametrize("call,give", [("fork", [0, -1, 2, 3]), ("fork", [0, 0, 2, 3]), ("resize", [-1, 0, -1, -1]), ("resize", [-1, 3, -1, -1])])
def test_what_is_given_back_need_not_be_sound(gto, call, give):
    """A slot that names no page is reported, the others are given back, and the call is carried out."""
    ctx, cfg, k, v = make(gto)
    do = lambda pool: gto.gto_pages_fork(ctx, pool, torch.tensor(give, **I32)) if call == "fork" else \
        gto.gto_pages_resize(ctx, pool, torch.tensor(give, **I32), k, v)
    whole = broken(gto, cfg)
    do(whole)
    assert gto.gto_decode_status(ctx) == 0 and whole["ref_count"][4].item() == 0
    want = numbers(whole)
    want["ref_count"][4] = 1                     # (its name is lost, its count stays)
    for no_page in (-1, 12, 2 ** 31 - 1):
        pool = broken(gto, cfg, page_table=((1, 1), no_page))
        do(pool)
        assert gto.gto_decode_status(ctx) == 8
        assert numbers(pool) == want


def test_what_the_page_calls_need_is_checked_before_anything_changes(gto):
    ctx, cfg, k, v = make(gto)
    for at in (dict(page_table=((1, 1), -1)), dict(page_table=((1, 1), 12)), dict(kv_len=(1, 9)), dict(held=(1, 6))):
        pool = broken(gto, cfg, **at)
        gto.gto_pages_fork(ctx, pool, torch.tensor([1, 1, 1, 3], **I32))     # 0 and 2 from 1, which is broken
        assert gto.gto_decode_status(ctx) == 8 and numbers(pool) == numbers(broken(gto, cfg, **at))
        for want in ([-1, 9, -1, -1], [-1, 20, -1, -1]):
            gto.gto_pages_resize(ctx, pool, torch.tensor(want, **I32), k, v)
            assert gto.gto_decode_status(ctx) == 8 and numbers(pool) == numbers(broken(gto, cfg, **at))
    # its own length says nothing about a sequence that becomes another's copy
    pool = broken(gto, cfg, kv_len=(1, 9))
    gto.gto_pages_fork(ctx, pool, torch.tensor([0, 0, 2, 3], **I32))
    assert gto.gto_decode_status(ctx) == 0
    assert pool["held"].tolist() == [3, 3, 0, 0] and pool["kv_len"].tolist() == [9, 9, 0, 0]
    assert pool["ref_count"].tolist() == [2, 2, 2] + [0] * 9
    # slots that stay and are not written are not looked at
    pool = broken(gto, cfg, page_table=((0, 0), 99))
    gto.gto_pages_resize(ctx, pool, torch.tensor([16, -1, -1, -1], **I32), k, v)
    assert gto.gto_decode_status(ctx) == 0 and pool["page_table"][0].tolist() == [99, 1, 2, 5, -1]


@pytest.mark.parametrize("at", [dict(page_table=((0, 1), 12)), dict(held=(0, 6)), dict(held=(0, -1))])
def test_compact_reports_a_row_that_is_broken_and_copies_it(gto, at):
    ctx, cfg, k, v = make(gto)
    pool = broken(gto, cfg, **at)
    table, ref, used = torch.zeros((4, 5), **I32), torch.zeros(12, **I32), torch.zeros(1, **I32)
    gto.gto_pages_compact(ctx, pool, k, v, table, ref, used)
    assert gto.gto_decode_status(ctx) == 8 and used.item() == 5
    assert torch.equal(table, pool["page_table"]) and torch.equal(ref, pool["ref_count"])


def test_too_few_pages_are_told_beside_other_faults(gto):
    """A caller that makes room and tries again has to be told, whatever else was wrong; and is told of that too."""
    cfg = gto.make_decode_config(S=4, T=4, n_q_heads=1, n_kv_heads=1, head_dim=16, page_size=4, n_pages=12, max_pages=5, dtype="f32",
                                 V_draft=64, V_target=64, logit_dtype="f32", flags=gto.GTO_DECODE_PAGES)
    ctx = gto.gto_decode_create(cfg, 0)
    k, v = (torch.zeros((12, 4, 1, 16), device=DEV) for _ in range(2))
    want = lambda *n: torch.tensor(n, **I32)
    draw = lambda heat: gto.gto_sample_tokens(ctx, torch.zeros((1, 64), device=DEV), dict(temperature=torch.tensor([heat], device=DEV)),
                                              torch.zeros(1, device=DEV), torch.zeros(1, **I32))
    status = lambda: [gto.gto_decode_status(ctx) for _ in range(3)]
    short = want(20, 20, 20, 20)                                       # 20 pages of 12
    pool = broken(gto, cfg)
    gto.gto_pages_resize(ctx, pool, short, k, v)
    assert status() == [9, 0, 0]
    pool = broken(gto, cfg, kv_len=(0, 13))
    gto.gto_pages_resize(ctx, pool, short, k, v)
    assert status() == [8, 9, 0]
    gto.gto_pages_resize(ctx, pool, short, k, v)
    draw(-1.0)
    assert status() == [8, 9, 0]                                       # (as ever: a bad index hides rows without a distribution)
    pool = broken(gto, cfg)
    gto.gto_pages_resize(ctx, pool, short, k, v)
    draw(-1.0)
    assert status() == [9, 5, 0]
    draw(1.0)
    assert status() == [0, 0, 0]


def test_a_step_that_does_not_look_after_pages_refuses_the_page_calls(gto):
    from paper_2509_22134_b200.runner import DecodeStep
    cfg = gto.make_decode_config(S=2, T=2, n_q_heads=1, n_kv_heads=1, head_dim=16, page_size=4, n_pages=12, max_pages=5, dtype="f32",
                                 V_draft=64, V_target=64, logit_dtype="f32")
    step = DecodeStep(cfg, 1, [])
    for call in (lambda: step.reserve(torch.zeros(2, **I32)), lambda: step.fork(torch.zeros(2, **I32)), step.compact):
        with pytest.raises(ValueError):
            call()
    step.close()
