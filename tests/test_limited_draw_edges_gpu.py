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


def cold_rows(rng, N, V):
    """fp32 rows whose likely logits lie 0 to 24 steps of fp32 below the largest, the others far below; the temperatures put
    999 halvings of a weight next to the middle between two such steps, on either side."""
    z = np.empty((N, V))
    heat = np.empty(N, np.float32)
    for i in range(N):
        top = np.float32(rng.choice([20.0, 60000.0, -3.0, 1.0, 3e-3, -7e5, 1e6]))
        step = abs(float(top) - float(np.nextafter(top, np.float32(-np.inf))))
        below = rng.choice([1, 2, 3, 4, 6, 8, 12, 16, 20])
        heat[i] = (below - 0.5 + rng.choice([-0.02, 0.02, 0.2])) * step / (999 * np.log(2.0))
        z[i] = float(top) - 1000 * step * (1 + rng.random(V))
        likely = rng.permutation(V)
        z[i, likely[:2]] = top
        for j in range(1, 25):
            z[i, likely[2 * j:2 * j + 2]] = float(top) - j * step
    z = z.astype(np.float32).astype(np.float64)
    return z, heat


@pytest.mark.parametrize("N", [3, 60, 170])
@pytest.mark.parametrize("limits", ["none", "k", "k and p", "k and min", "p", "all"])
def test_weights_that_vanish_within_a_few_steps_of_fp32(gto, limits, N):
    rng = np.random.default_rng(33)
    V = 8192
    z, heat = cold_rows(rng, N, V)
    s = dict(temperature=heat)
    if "k" in limits or limits == "all":
        s["top_k"] = rng.integers(1500, 7000, N).astype(np.int32)
    if "p" in limits or limits == "all":
        s["top_p"] = (1 - 0.3 * rng.random(N)).astype(np.float32)
    if "min" in limits or limits == "all":
        s["min_p"] = np.full(N, 1e-3, np.float32)
    for u in (rng.random(N).astype(np.float32), np.full(N, 0.5 + 2.0 ** -23, np.float32), np.full(N, 0.5 - 2.0 ** -23, np.float32)):
        ctx, out = run(gto, z, s, u, "f32")
        assert gto.gto_decode_status(ctx) == 0
        check(z, s, u, out)


@pytest.mark.parametrize("limits", ["none", "k", "k and p"])
def test_trees_whose_weights_vanish_within_a_few_steps_of_fp32(gto, limits):
    rng = np.random.default_rng(34)
    S, g, D, V = 20, 12, 3, 8192
    c = verify_case(rng, S, g, D, V, V, "f32")
    for i in range(S):
        rows, heat = cold_rows(rng, 1, V)
        c["target"][i] = [rng.permutation(rows[0]) for _ in range(1 + g)]
        c["temperature"][i] = heat[0]
        for n in range(g):                     # each node one of its context's two largest
            context = c["target"][i, 1 + c["parent"][i, n]]
            c["token"][i, n] = np.flatnonzero(context == context.max())[n % 2]
    c["u_node"] = (0.5 + rng.choice([-1, 1], (S, g)) * 2.0 ** -rng.integers(2, 22, (S, g))).astype(np.float32)
    s = dict(temperature=c["temperature"].astype(np.float32))
    if "k" in limits:
        s["top_k"] = rng.integers(1500, 7000, S).astype(np.int32)
    if "p" in limits:
        s["top_p"] = np.full(S, 0.999, np.float32)
    ctx, out, _ = run_tree(gto, c, s, D, V, V, "f32")
    assert gto.gto_decode_status(ctx) == 0
    check_tree(c, s, out, D)
