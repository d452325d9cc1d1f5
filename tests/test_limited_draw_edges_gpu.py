"""gto_sample_tokens and gto_verify_tree_limited where an exchange between CTAs, or an exponent, is at its edge."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from test_decode_gpu import verify_case
from test_limited_draw_gpu import check, check_tree, logits, run, run_tree, settings

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


@pytest.mark.parametrize("dtype,V,N", [("bf16", 8, 1), ("f16", 8, 74), ("f32", 4, 30), ("bf16", 64, 37), ("f32", 32772, 20), ("bf16", 65544, 37)])
def test_rows_that_are_read_at_once_and_rows_that_are_not_read(gto, dtype, V, N):
    """The CTAs of a cluster tell each other what they have read right after their start, or have read nothing."""
    rng = np.random.default_rng(V + N)
    z = dc.round_to(logits(rng, "normal", N, V), dtype)
    s, u = settings(rng, "all", N, V), rng.random(N).astype(np.float32)
    s["temperature"][3::5] = [-1.0, np.nan][N % 2]
    rows = np.arange(N)
    rows[4::5] = N
    ctx, first = run(gto, z, s, u, dtype, rows=rows)
    assert gto.gto_decode_status(ctx) == (8 if N > 4 else 0)
    none = (np.arange(N) % 5 == 3) | (rows == N)
    assert (first["token"][none] == -1).all() and (first["n_kept"][none] == 0).all()
    keep = ~none
    check(z, {k: v[keep] for k, v in s.items()}, u[keep], {k: v[keep] for k, v in first.items()}, rows=np.arange(N)[keep])
    for turn in range(20):
        _, again = run(gto, z, s, u, dtype, ctx=ctx, rows=rows)
        assert all(np.array_equal(again[k], first[k]) for k in first)


@pytest.mark.parametrize("dtype,V", [("bf16", 8), ("f32", 4), ("f16", 1000)])
def test_trees_over_short_rows_and_trees_that_read_none(gto, dtype, V):
    rng = np.random.default_rng(V)
    S, g, D = 40, 3, 2
    c = verify_case(rng, S, g, D, V, V, dtype)
    s = settings(rng, "all", S, V)
    s["temperature"][2::3] = np.inf
    ctx, first, args = run_tree(gto, c, s, D, V, V, dtype)
    assert gto.gto_decode_status(ctx) == 5
    assert (first["accept_len"][2::3] == 0).all() and (first["token"][2::3] == -1).all()
    check_tree(c, s, first, D)
    out = gto.alloc_verdict(ctx.cfg, DEV)
    for turn in range(20):
        gto.gto_verify_tree_limited(ctx, *args, out)
        assert all(np.array_equal(out[k].cpu().numpy(), first[k]) for k in first)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_left_rows_of_which_some_are_not_read(gto, dtype):
    """The second kernel of a batch: clusters with several rows, with one, and with none."""
    rng = np.random.default_rng(31)
    N, V = 1300, 2048
    z = dc.round_to(logits(rng, "flat", 50, V), dtype)
    rows, u = rng.integers(0, 50, N), rng.random(N).astype(np.float32)
    s = dict(temperature=np.full(N, 0.8, np.float32), top_p=np.full(N, 0.9, np.float32))
    ctx = None
    for n in (1300, 300, 149):
        for few in (False, True):  # few: all but three rows are greedy, and nothing is left of them
            part = {k: v[:n].copy() for k, v in s.items()}
            if few:
                part["temperature"][3:] = 0.0
            part["temperature"][10::7] = -1.0
            ctx, out = run(gto, z, part, u[:n], dtype, ctx=ctx, rows=rows[:n], S=N)
            assert gto.gto_decode_status(ctx) == 5
            assert (out["token"][10::7] == -1).all()
            check(z, part, u[:n], out, rows=rows[:n])


def test_more_left_rows_than_are_listed_call_after_call(gto):
    """All CTAs of the second kernel read how many rows are left; the last one sets the number back for the next call."""
    rng = np.random.default_rng(32)
    V, R, N = 1024, 16, 4500
    z = torch.from_numpy(dc.round_to(logits(rng, "flat", R, V), "f16")).to(DEV, torch.float16)
    rows, u = rng.integers(0, R, N), rng.random(N).astype(np.float32)
    s = dict(temperature=np.full(N, 1.0, np.float32), top_p=(0.6 + 0.39 * rng.random(N)).astype(np.float32))
    ctx, first = run(gto, z, s, u, "f16", rows=rows, S=N)
    assert gto.gto_decode_status(ctx) == 0
    check(z.double().cpu().numpy(), s, u, first, rows=rows)
    for turn in range(60):
        n = N if turn % 3 else 100
        _, again = run(gto, z, {k: v[:n] for k, v in s.items()}, u[:n], "f16", ctx=ctx, rows=rows[:n])
        assert all(np.array_equal(again[k], first[k][:n]) for k in first), turn
    assert gto.gto_decode_status(ctx) == 0
