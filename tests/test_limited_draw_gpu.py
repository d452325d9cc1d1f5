"""gto_sample_tokens and gto_verify_tree_limited against the fp64 oracle."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import limits_oracle as lim
from test_decode_gpu import verify_case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# The inputs put no decision where two fp64 orders of summation (1e5 terms) could differ.
CLEAR = 1e-12
# A log-probability is rounded once to fp32; the mass under it may be a sum of fp32 weights, off by at most 4e-6 of itself
# (5.7e-6 with the fp64 logarithm's argument on both sides of the quotient is not reached: the weight above is fp64).
LOGP = lambda x: 2.0 ** -24 * abs(x) + 4.1e-6


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    return t if dtype is None else t.to(dtype)


def logits(rng, kind, N, V):
    if kind == "power":       # probabilities that fall with a power of the rank, as a language model's
        return 14 - rng.uniform(1.05, 2.0, (N, 1)) * np.log(1 + V * rng.random((N, V))) + 0.3 * rng.normal(size=(N, V))
    if kind == "normal":
        return 2 * rng.normal(size=(N, V))
    if kind == "flat":
        return 0.05 * rng.normal(size=(N, V)) - 3
    if kind == "steps":       # few values: ties everywhere, also of 0 and -0
        return np.round(rng.normal(size=(N, V)) * 1.2) * 0.5 * rng.choice([1.0, -1.0], size=(N, V))
    z = 3 * rng.normal(size=(N, V))
    if kind == "masked":      # most of the vocabulary is ruled out, some rows have one token left, some masks are the lowest value
        z[rng.random((N, V)) < 0.9] = -np.inf
        z[::5] = -np.inf
        z[::3][z[::3] == -np.inf] = -65504.0
        z[np.arange(N), rng.integers(0, V, N)] = 1.0
        return z
    assert kind == "far"      # one token far above all others
    z[np.arange(N), rng.integers(0, V, N)] += 300
    return z


def settings(rng, kind, N, V):
    s = dict(temperature=rng.uniform(0.4, 1.5, N))
    if kind in ("k", "mixed", "all"):
        s["top_k"] = np.exp(rng.uniform(0, np.log(V) + 0.5, N)).astype(np.int64)
    if kind in ("p", "mixed", "all"):
        s["top_p"] = 1 - np.exp(rng.uniform(np.log(1e-4), 0, N))
    if kind in ("min", "mixed", "all"):
        s["min_p"] = np.exp(rng.uniform(np.log(1e-6), 0, N))
    if kind == "mixed":
        s["temperature"][1::4] = 0
        s["top_k"][::2] = [0, -3][N % 2]
        s["top_p"][::3] = 1.0
        s["min_p"][1::3] = 0.0
    return {k: v.astype(np.int32 if k == "top_k" else np.float32) for k, v in s.items()}


def run(gto, z, s, u, dtype, ctx=None, rows=None, stream=None, S=None):
    N, V = len(u), z.shape[1]
    ctx = ctx or gto.gto_decode_create(gto.make_decode_config(S=S or N, V_draft=V, V_target=V, logit_dtype=dtype), 0)
    z = z if torch.is_tensor(z) else dev(z, dc.TORCH[dtype])
    out = dict(token=torch.full((N,), -77, dtype=torch.int32, device=DEV), logp=torch.full((N,), 7.0, device=DEV),
               n_kept=torch.full((N,), -77, dtype=torch.int32, device=DEV))
    gto.gto_sample_tokens(ctx, z, {k: dev(v) for k, v in s.items()}, dev(np.asarray(u, np.float32)), out["token"], logp=out["logp"],
                          n_kept=out["n_kept"], rows=None if rows is None else dev(np.asarray(rows, np.int32)), stream=stream)
    return ctx, {k: v.cpu().numpy() for k, v in out.items()}


def check(z, s, u, out, rows=None, least=0.9):
    """z: fp64 values that the type can hold."""
    clear = 0
    for i in range(len(u)):
        one = {k: (int if k == "top_k" else float)(v[i]) for k, v in s.items()}
        token, logp, n, margin = lim.sample(z[i if rows is None else rows[i]], u=float(np.float32(u[i])), **one)
        if margin < CLEAR:
            continue
        clear += 1
        what = (i, one, float(u[i]))
        assert out["n_kept"][i] == n, what
        assert out["token"][i] == token, what
        assert abs(out["logp"][i] - logp) <= LOGP(logp), what
    assert clear >= least * len(u)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("limits", ["none", "k", "p", "min", "all", "mixed"])
@pytest.mark.parametrize("kind", ["power", "normal", "flat", "steps", "masked", "far"])
def test_sample(gto, kind, limits, dtype):
    for N, V in ((24, 512), (7, 8), (33, 1000), (5, 32000)):
        rng = np.random.default_rng(N + V)
        z = dc.round_to(logits(rng, kind, N, V), dtype)
        s, u = settings(rng, limits, N, V), rng.random(N).astype(np.float32)
        ctx, out = run(gto, z, s, u, dtype)
        assert gto.gto_decode_status(ctx) == 0
        # (steps: equal weights whose sums meet a multiple of u or top_p exactly are no clear decision)
        check(z, s, u, out, least=0.5 if kind in ("steps", "masked") else 0.9)


@pytest.mark.parametrize("dtype,V", [("bf16", 128256), ("f32", 151936), ("f16", 65536), ("bf16", 786432), ("f32", 393216)])
@pytest.mark.parametrize("N", [1, 6, 50, 170])
def test_sample_long_rows(gto, dtype, V, N):
    if N > 6 and V > 200000:
        N = 9
    rng = np.random.default_rng(N)
    z = np.empty((N, V))
    for i in range(N):
        z[i] = logits(rng, ["power", "power", "normal", "flat", "steps"][i % 5], 1, V)
    z = dc.round_to(z, dtype)
    for limits in ("mixed", "none", "all")[:3 if N <= 6 else 2]:
        s, u = settings(rng, limits, N, V), rng.random(N).astype(np.float32)
        ctx, out = run(gto, z, s, u, dtype)
        assert gto.gto_decode_status(ctx) == 0
        check(z, s, u, out, least=0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sample_at_the_borders_of_the_settings(gto, dtype):
    V = 4096
    rng = np.random.default_rng(5)
    base = dc.round_to(2 * rng.normal(size=V), dtype)
    rows = []
    for k in (1, 2, V - 1, V, V + 1, 2 ** 31 - 1, 0, -1, -2 ** 31):
        rows.append(dict(top_k=k))
    for p in (0.0, -1.0, 1e-30, 0.5, 1 - 2.0 ** -24, 1.0, 1.5, np.inf, -np.inf):
        rows.append(dict(top_p=p))
    for p in (0.0, -1.0, 1e-30, 1e-44, 0.5, 1 - 2.0 ** -24, 1.0, 1.5, np.inf, -np.inf):
        rows.append(dict(min_p=p))
    for t in (0.0, 1e-44, 1e-30, 1e-3, 300.0, 3e38):
        rows.append(dict(temperature=t))
        rows.append(dict(temperature=t, top_p=0.7))
        rows.append(dict(temperature=t, top_k=40, min_p=0.1))
    u = [0.0, 2.0 ** -149, 0.25, 1 - 2.0 ** -24, 1.0, -3.0, 7.0]
    both = [(r, x) for r in rows for x in u]
    s = {n: np.array([r.get(n, d) for r, _ in both], t) for n, d, t in
         (("temperature", 1.0, np.float32), ("top_k", 0, np.int32), ("top_p", 1.0, np.float32), ("min_p", 0.0, np.float32))}
    z, us = np.tile(base, (len(both), 1)), np.array([x for _, x in both], np.float32)
    ctx, out = run(gto, z, s, us, dtype)
    assert gto.gto_decode_status(ctx) == 0
    check(z, s, us, out, least=0.85)
    nan = np.full(3, np.nan, np.float32)   # a uniform that is none counts as 0
    one = dict(temperature=np.ones(3, np.float32))
    assert np.array_equal(run(gto, z[:3], one, nan, dtype)[1]["token"], run(gto, z[:3], one, 0 * us[:3], dtype)[1]["token"])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("V", [2048, 40000])
def test_sample_rows_of_equal_logits(gto, dtype, V):
    """All tokens at the border: the lowest ids stay, exactly as many as the limit says."""
    z = np.full((8, V), 1.5)
    z[4:, ::2] = -65504.0
    s = dict(temperature=np.full(8, 0.7, np.float32), top_k=np.array([0, 700, 0, 900, 0, 700, 0, 900], np.int32),
             top_p=np.array([1, 1, 0.25, 0.5, 1, 1, 0.25, 0.5], np.float32))
    u = np.array([0.3] * 4 + [0.77] * 4, np.float32)
    ctx, out = run(gto, z, s, u, dtype)
    half = V // 2
    assert out["n_kept"].tolist() == [V, 700, V // 4, 450, V, 700, half // 4, 450]
    at = lambda n, x: int(np.floor(np.float64(np.float32(x)) * n))
    want = [at(n, 0.3) for n in (V, 700, V // 4, 450)] + [2 * at(n, 0.77) + 1 for n in (half, 700, half // 4, 450)]
    assert out["token"].tolist() == want


def test_sample_from_given_rows_of_a_wider_matrix(gto):
    rng = np.random.default_rng(3)
    V, R, N = 1000, 9, 40
    wide = dev(dc.round_to(logits(rng, "power", R, V + 56), "bf16"), torch.bfloat16)
    rows = rng.integers(0, R, N)
    s, u = settings(rng, "mixed", N, V), rng.random(N)
    ctx, out = run(gto, wide[:, 16:16 + V], s, u, "bf16", rows=rows, S=64)
    z = wide[:, 16:16 + V].double().cpu().numpy()
    check(z, s, u.astype(np.float32), out, rows=rows)
    bad = rows.copy()
    bad[[0, 7, 39]] = [-1, R, 2 ** 31 - 1]
    assert gto.gto_decode_status(ctx) == 0
    _, got = run(gto, wide[:, 16:16 + V], s, u, "bf16", ctx=ctx, rows=bad)
    assert gto.gto_decode_status(ctx) == 8
    keep = np.ones(N, bool)
    keep[[0, 7, 39]] = False
    for k in out:
        assert np.array_equal(got[k][keep], out[k][keep])
    assert (got["token"][~keep] == -1).all() and (got["logp"][~keep] == 0).all() and (got["n_kept"][~keep] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_sample_reports_rows_that_hold_no_distribution(gto, dtype):
    V = 4096
    rng = np.random.default_rng(4)
    z = dc.round_to(rng.normal(size=(12, V)), dtype)
    z[1, 4000], z[2, 5], z[3] = np.nan, np.inf, -np.inf
    z[4, :] = np.nan
    s = dict(temperature=np.ones(12, np.float32), top_p=np.full(12, 0.9, np.float32), min_p=np.full(12, 0.01, np.float32))
    s["temperature"][5:8] = [-1.0, np.nan, np.inf]
    s["top_p"][8], s["min_p"][9] = np.nan, np.nan
    u = rng.random(12).astype(np.float32)
    ctx, out = run(gto, z, s, u, dtype)
    assert gto.gto_decode_status(ctx) == 5
    assert (out["token"][1:10] == -1).all() and (out["n_kept"][1:10] == 0).all() and (out["logp"][1:10] == 0).all()
    check(z, s, u, out)


def test_sample_follows_the_distribution(gto):
    """A regular grid of u over one row: every token that stays has its share, to one grid step."""
    rng = np.random.default_rng(6)
    V, N = 4096, 8192
    z = dc.round_to(logits(rng, "power", 1, V), "bf16")
    s = {k: np.full(N, v, t) for k, v, t in (("temperature", 0.9, np.float32), ("top_k", 300, np.int32), ("top_p", 0.95, np.float32))}
    u = (np.arange(N) + 0.5) / N
    ctx, out = run(gto, z, s, u, "bf16", rows=np.zeros(N, int))
    w, ids, _ = lim.kept(z[0], float(np.float32(0.9)), 300, float(np.float32(0.95)))
    p = np.zeros(V)
    p[ids] = w[ids] / w[ids].sum()
    assert np.abs(np.bincount(out["token"], minlength=V) / N - p).max() <= 1.0 / N + 1e-6


def test_sample_in_a_graph_on_another_stream_and_twice_the_same(gto):
    rng = np.random.default_rng(7)
    N, V = 40, 8192
    z = dev(dc.round_to(logits(rng, "power", N, V), "f16"), torch.float16)
    s, u = settings(rng, "mixed", N, V), rng.random(N).astype(np.float32)
    cfg = gto.make_decode_config(S=N, V_draft=V, V_target=V, logit_dtype="f16")
    ctx = gto.gto_decode_create(cfg, 0)
    d, du = {k: dev(v) for k, v in s.items()}, dev(u)
    out = [torch.zeros(N, dtype=torch.int32, device=DEV), torch.zeros(N, device=DEV), torch.zeros(N, dtype=torch.int32, device=DEV)]
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    gto.gto_sample_tokens(ctx, z, d, du, out[0], out[1], out[2], stream=side)
    side.synchronize()
    first = [t.clone() for t in out]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gto.gto_sample_tokens(ctx, z, d, du, *out)
    for turn in range(3):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, first))
    u2 = rng.random(N).astype(np.float32)           # the same graph with other contents
    s2 = settings(rng, "all", N, V)
    du.copy_(dev(u2))
    for k in d:
        d[k].copy_(dev(s2[k]))
    graph.replay()
    torch.cuda.synchronize()
    check(z.double().cpu().numpy(), s2, u2, dict(token=out[0].cpu().numpy(), logp=out[1].cpu().numpy(), n_kept=out[2].cpu().numpy()))
    del graph


# ------------------------------------------------------------------ trees

def run_tree(gto, c, s, D, V, Vd, dtype):
    S, g = c["parent"].shape
    cfg = gto.make_decode_config(S=S, g=g, D=D, V_draft=Vd, V_target=V, logit_dtype=dtype)
    ctx = gto.gto_decode_create(cfg, 0)
    out = gto.alloc_verdict(cfg, DEV)
    for t in out.values():
        t.fill_(-77)
    tree = dict(node_token=dev(c["token"]), node_parent=dev(c["parent"]))
    if c["n_nodes"] is not None:
        tree["n_nodes"] = dev(np.array(c["n_nodes"], np.int32))
    args = (tree, dev(c["target"], dc.TORCH[dtype]), None if c["d2t"] is None else dev(c["d2t"]), {k: dev(v) for k, v in s.items()},
            dev(c["u_node"]), dev(c["u_bonus"]))
    gto.gto_verify_tree_limited(ctx, *args, out)
    return ctx, {k: v.cpu().numpy() for k, v in out.items()}, args


def check_tree(c, s, out, D, least=0.9):
    clear = 0
    S = len(c["parent"])
    for i in range(S):
        g = c["parent"].shape[1] if c["n_nodes"] is None else c["n_nodes"][i]
        one = {k: (int if k == "top_k" else float)(v[i]) for k, v in s.items()}
        path, ids, last, margin = lim.verify(c["parent"][i][:g], c["token"][i][:g], 1 + np.arange(g), c["target"][i],
                                             u_node=c["u_node"][i].astype(float), u_bonus=float(c["u_bonus"][i]), D=D, d2t=c["d2t"], **one)
        if margin < CLEAR:
            continue
        clear += 1
        assert out["accept_len"][i] == len(path), (i, one)
        assert list(out["path_node"][i]) == path + [-1] * (D - len(path))
        assert list(out["token"][i]) == ids + [last] + [-1] * (D - len(path)), (i, one)
    assert clear >= least * S


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("limits", ["none", "k", "p", "min", "mixed"])
@pytest.mark.parametrize("S,g,D,V,Vd", [
    (5, 12, 3, 512, 512), (33, 60, 7, 1000, 200), (3, 1, 1, 16, 16), (4, 0, 1, 2048, 2048), (6, 128, 16, 4104, 4104),
    (2, 40, 5, 32000, 8000)])
def test_verify_limited(gto, S, g, D, V, Vd, limits, dtype):
    rng = np.random.default_rng(S + V)
    c = verify_case(rng, S, g, D, V, Vd, dtype)
    s = settings(rng, limits, S, V)
    ctx, out, _ = run_tree(gto, c, s, D, V, Vd, dtype)
    assert gto.gto_decode_status(ctx) == 0
    check_tree(c, s, out, D)


def test_verify_limited_flat_rows_ragged_trees_and_repeated_siblings(gto):
    rng = np.random.default_rng(11)
    S, g, D, V = 40, 30, 6, 8192
    n = rng.integers(0, g + 1, S)
    n[:3] = [0, 1, g]
    c = verify_case(rng, S, g, D, V, V, "bf16", n_nodes=n)
    c["token"][:, 1::3] = c["token"][:, ::3]
    c["target"][::2] = dc.round_to(0.01 * rng.normal(size=c["target"][::2].shape), "bf16")
    c["target"][1::4][..., ::7] = -np.inf
    for limits in ("none", "k", "p", "mixed"):
        s = settings(rng, limits, S, V)
        ctx, out, _ = run_tree(gto, c, s, D, V, V, "bf16")
        assert gto.gto_decode_status(ctx) == 0
        check_tree(c, s, out, D)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_limits_it_is_the_plain_verification(gto, dtype):
    rng = np.random.default_rng(12)
    S, g, D, V = 50, 60, 7, 4096
    c = verify_case(rng, S, g, D, V, V, dtype)
    off = dict(temperature=c["temperature"], top_k=np.zeros(S, np.int32), top_p=np.ones(S, np.float32), min_p=np.zeros(S, np.float32))
    ctx, out, args = run_tree(gto, c, off, D, V, V, dtype)
    plain = gto.alloc_verdict(ctx.cfg, DEV)
    gto.gto_verify_tree(ctx, args[0], args[1], None, args[3]["temperature"], args[4], args[5], plain)
    for k in out:
        assert np.array_equal(out[k], plain[k].cpu().numpy())


def test_verify_limited_reports_bad_rows_settings_and_indices(gto):
    rng = np.random.default_rng(13)
    S, g, D, V = 10, 12, 3, 1024
    c = verify_case(rng, S, g, D, V, V, "f32")
    s = dict(temperature=np.ones(S, np.float32), top_p=np.full(S, 0.95, np.float32))
    c["target"][1, 0, 5], c["target"][2, 0] = np.nan, -np.inf
    s["temperature"][3], s["top_p"][4] = np.inf, np.nan
    ctx, out, _ = run_tree(gto, c, s, D, V, V, "f32")
    assert gto.gto_decode_status(ctx) == 5
    assert (out["accept_len"][1:5] == 0).all() and (out["token"][1:5] == -1).all() and (out["path_node"][1:5] == -1).all()
    check_tree(c, s, out, D)
    c["token"][6, 3], c["parent"][7, 2], c["n_nodes"] = V, 5, np.array([g] * 8 + [g + 1, -1])
    ctx, out, _ = run_tree(gto, c, s, D, V, V, "f32")
    assert gto.gto_decode_status(ctx) == 8
    c["parent"][6, 3] = c["parent"][7, 2] = 99      # what is not followed is nobody's child
    c["n_nodes"][8:] = 0
    check_tree(c, s, out, D)


def test_verify_limited_in_the_layout_of_the_reward_pass(gto):
    """Target rows by depth and frontier slot against the same rows by node."""
    import harness
    from paper_2509_22134_b200 import synth
    w = synth.Workload("t", B=16, V_draft=512, V_target=2048, D=4, k=4, g=20, dtype="f32", seed=8, sigma_t=1.0, boost=8.0)
    p, data = harness.run_pass(w, DEV)
    S, N = w.B, 60
    names = ("node_token", "node_parent", "node_depth", "node_slot")
    tree = {n: p.tree[n][0].contiguous().repeat(N, 1) for n in names}
    target, d2t = data["target"][0].contiguous().repeat(N, 1, 1), data["d2t"]
    cfg = lambda flags: gto.make_decode_config(S=S * N, g=w.g, D=w.D, k=w.k, V_draft=w.V_draft, V_target=w.V_target,
                                               logit_dtype=w.dtype, flags=flags)
    gen = torch.Generator(DEV).manual_seed(1)
    limits = dict(temperature=0.6 + torch.rand(S * N, generator=gen, device=DEV), top_p=torch.rand(S * N, generator=gen, device=DEV))
    u, ub = torch.rand((S * N, w.g), generator=gen, device=DEV), torch.rand(S * N, generator=gen, device=DEV)
    ctx = gto.gto_decode_create(cfg(gto.GTO_DECODE_CONTEXT_ROWS), 0)
    out = gto.alloc_verdict(ctx.cfg, DEV)
    gto.gto_verify_tree_limited(ctx, tree, target, d2t, limits, u, ub, out)
    assert gto.gto_decode_status(ctx) == 0
    depth, slot = tree["node_depth"].long(), tree["node_slot"].long()
    has = (slot >= 0) & (depth < w.D)
    at = torch.where(has, 1 + (depth - 1) * w.k + slot, 0)
    by_node = torch.cat([target[:, :1], target[torch.arange(S * N, device=DEV)[:, None], at]], 1).contiguous()
    plain = gto.gto_decode_create(cfg(0), 0)
    want = gto.alloc_verdict(plain.cfg, DEV)
    gto.gto_verify_tree_limited(plain, tree, by_node, d2t, limits, u, ub, want)
    leaf = torch.gather(want["path_node"].long(), 1, (want["accept_len"].long() - 1).clamp(min=0)[:, None])[:, 0].clamp(min=0)
    ends = (want["accept_len"] > 0) & ~has[torch.arange(S * N, device=DEV), leaf]   # no row there: no token after it
    assert bool(ends.any()) and bool((~ends).any())
    want["token"][torch.nonzero(ends)[:, 0], want["accept_len"][ends].long()] = -1
    # (a node without a row has no children among the nodes)
    for k in out:
        assert torch.equal(out[k], want[k]), k


def test_sample_where_nearly_all_rows_need_more_than_a_list(gto):
    """More rows than are listed for the second kernel: it finds them by their marks; the next call begins anew."""
    rng = np.random.default_rng(21)
    V, R, N = 2048, 40, 6000
    z = dc.round_to(logits(rng, "flat", R, V), "f16")
    rows, u = rng.integers(0, R, N), rng.random(N).astype(np.float32)
    s = settings(rng, "p", N, V)
    s["top_p"] = (0.3 + 0.69 * rng.random(N)).astype(np.float32)
    ctx, out = run(gto, z, s, u, "f16", rows=rows)
    assert gto.gto_decode_status(ctx) == 0
    check(z, s, u, out, rows=rows)
    for n in (6000, 4097, 4096, 300):
        _, again = run(gto, z, {k: v[:n] for k, v in s.items()}, u[:n], "f16", ctx=ctx, rows=rows[:n])
        for k in out:
            assert np.array_equal(again[k], out[k][:n])


def test_two_contexts_draw_on_two_streams_at_once(gto):
    rng = np.random.default_rng(22)
    N, V = 200, 16384
    cfg = gto.make_decode_config(S=N, V_draft=V, V_target=V, logit_dtype="bf16")
    sets = []
    for kind in ("power", "flat"):
        z = dev(dc.round_to(logits(rng, kind, N, V), "bf16"), torch.bfloat16)
        s, u = {k: dev(v) for k, v in settings(rng, "mixed", N, V).items()}, dev(rng.random(N).astype(np.float32))
        outs = [[torch.full((N,), -77, dtype=t, device=DEV) for t in (torch.int32, torch.float32, torch.int32)] for _ in range(8)]
        sets.append((gto.gto_decode_create(cfg, 0), torch.cuda.Stream(DEV), z, s, u, outs))
    torch.cuda.synchronize()
    for turn in range(8):
        for ctx, stream, z, s, u, outs in sets:
            gto.gto_sample_tokens(ctx, z, s, u, *outs[turn], stream=stream)
    torch.cuda.synchronize()
    for ctx, stream, z, s, u, outs in sets:
        assert gto.gto_decode_status(ctx) == 0
        for o in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
        check(z.double().cpu().numpy(), {k: v.cpu().numpy() for k, v in s.items()}, u.cpu().numpy(),
              dict(zip(("token", "logp", "n_kept"), (t.cpu().numpy() for t in outs[0]))))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("alone", [False, True])
def test_verify_limited_refuses_a_token_that_is_nearly_all(gto, dtype, alone):
    """What is left of such a row is a millionth of it, and nothing where the token stood."""
    rng = np.random.default_rng(23)
    S, V = 16, 8192
    c = verify_case(rng, S, 1, 1, V, V, dtype)
    z = 0.5 * rng.normal(size=(S, 2, V))
    heavy = rng.integers(0, V, S)
    for i in range(S):
        if alone:
            z[i, 0, max(heavy[i] - 300, 0):heavy[i] + 300] = -np.inf
        z[i, 0, heavy[i]] = 21.0
    c["target"] = dc.round_to(z, dtype)
    c["token"][:, 0], c["parent"][:, 0] = heavy, -1
    c["u_node"] = np.full((S, 1), 1 - 2.0 ** -24, np.float32)
    s = dict(temperature=np.ones(S, np.float32), top_k=rng.integers(3000, 7000, S).astype(np.int32))
    ctx, out, _ = run_tree(gto, c, s, 1, V, V, dtype)
    assert gto.gto_decode_status(ctx) == 0
    assert (out["accept_len"] == 0).all() and (out["token"][:, 0] != heavy).all()
    # (the rest is 1e-6 of the whole, whose sums are good to 1e-15: decisions clearer than 1e-8 of it are told)
    clear = 0
    for i in range(S):
        _, _, last, margin = lim.verify(c["parent"][i], c["token"][i], 1 + np.arange(1), c["target"][i], u_node=c["u_node"][i].astype(float),
                                        u_bonus=float(c["u_bonus"][i]), D=1, d2t=None, temperature=1.0, top_k=int(s["top_k"][i]))
        if margin > 1e-8:
            clear += 1
            assert out["token"][i, 0] == last
    assert clear >= 12


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("N", [2, 60, 160])
def test_sample_rows_whose_logits_lie_next_to_one_another(gto, dtype, N):
    """More tokens at one distance from the largest logit than a counter holds; top-k among them, with and without the others."""
    rng = np.random.default_rng(24)
    V = 16384
    z = dc.round_to(0.5 + 0.005 * rng.integers(-1, 2, (N, V)) + 1e-4 * rng.integers(-30, 30, (N, V)), dtype)
    u = rng.random(N).astype(np.float32)
    k = rng.integers(5000, 16000, N).astype(np.int32)
    for more in (dict(), dict(min_p=1e-6), dict(top_p=0.8), dict(top_p=0.999, min_p=0.5)):
        s = dict(temperature=np.full(N, 0.9, np.float32), top_k=k, **{n: np.full(N, x, np.float32) for n, x in more.items()})
        ctx, out = run(gto, z, s, u, dtype)
        assert gto.gto_decode_status(ctx) == 0
        check(z, s, u, out, least=0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("N", [3, 80])
def test_sample_cold_rows_with_long_tails(gto, dtype, N):
    """All the mass in a few tokens, the values far apart: no estimate by distance tells where the mass is."""
    rng = np.random.default_rng(25)
    V = 24000
    z = dc.round_to(np.clip(5 * rng.standard_t(1.5, (N, V)), -6e4, 6e4), dtype)
    u = rng.random(N).astype(np.float32)
    for heat in (1e-5, 1e-3, 0.1):
        s = dict(temperature=np.full(N, heat, np.float32), top_k=rng.integers(2000, 20000, N).astype(np.int32),
                 top_p=(1 - 1e-3 * rng.random(N)).astype(np.float32))
        ctx, out = run(gto, z, s, u, dtype)
        assert gto.gto_decode_status(ctx) == 0
        check(z, s, u, out)
