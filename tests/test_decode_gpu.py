"""The decoding step over a draft tree, call by call against the fp64 oracle, through the C ABI."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import decode_oracle as dec
from oracle import gto_oracle as orc
from paper_2509_22134_b200 import synth

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


# ------------------------------------------------------------------ gto_kv_append

def append_tolerance(dtype, x):
    """fp32 arithmetic on values up to |x| (rotation: two products and a sum, norm: a sum of head_dim squares, a root,
    two products; cos and sin to 2^-23; angle reduced to 2^-25 turns = 1.9e-7 rad): 2^-20 relative to the pair's size
    covers the sum of these; then one rounding to the type."""
    return np.abs(x).max() * 2.0 ** -20 + dc.HALF_STEP[dtype] * np.abs(x)


APPEND = [
    # q_lens, kv_lens, (hq, hkv, dh), page, g, D, n_nodes, rope, interleaved, norm
    ([1], [1], (4, 2, 64), 16, 0, 1, None, 64, False, False),               # the first token of a sequence
    ([1, 1, 1], [100001, 5, 17], (4, 2, 128), 16, 0, 1, None, 128, False, False),   # a far position
    ([5, 0, 33], [5, 9, 70], (8, 8, 64), 8, 0, 1, None, 64, True, False),   # a prompt, a sequence without a chunk
    ([13, 14], [40, 300], (6, 2, 128), 32, 12, 4, None, 64, False, True),   # trees, part of the head rotated, norms
    ([13, 3, 0], [13, 64, 7], (4, 4, 96), 5, 12, 4, [12, 0, 0], 96, False, True),  # odd page, head of 96, ragged trees
    ([70], [200], (2, 1, 256), 64, 70, 6, None, 256, True, True),           # lead 0: the tree hangs below the cache
    ([2, 1], [9, 8], (3, 1, 16), 4, 0, 1, None, 0, False, False),           # nothing rotated
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(gto, case, dtype):
    q_lens, kv_lens, (hq, hkv, dh), page, g, D, n_nodes, rope, inter, norm = APPEND[case]
    c = dc.Case(q_lens, kv_lens, hq, hkv, dh, page, dtype, g, D, n_nodes, seed=case, head_major=case % 2 == 1, poison=3.0)
    qkv = dc.round_to(c.rng.normal(size=(c.T, hq + 2 * hkv, dh)), dtype)
    f = 500000.0 ** (-np.arange(rope // 2) / max(rope // 2, 1))
    w = [dc.round_to(1 + 0.3 * c.rng.normal(size=dh), dtype) if norm else None for _ in range(2)]
    ctx = c.ctx(gto, rope_dims=rope, flags=gto.GTO_DECODE_ROPE_INTERLEAVED if inter else 0)
    x = c.tensor(qkv)
    q_out = torch.full((c.T, hq, dh), 7.0, dtype=x.dtype, device=DEV)
    dw = [None if v is None else c.tensor(v) for v in w]
    gto.gto_kv_append(ctx, c.batch, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q_out, c.dk, c.dv,
                      torch.tensor(f, device=DEV), dw[0], dw[1])
    assert gto.gto_decode_status(ctx) == 0
    want_q, want_k, want_v = dec.append(c.host, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], c.k, c.v, page, f, g,
                                        inter, w[0], w[1])
    assert torch.equal(c.dv.double().cpu(), torch.tensor(want_v))           # values are copies, all else untouched
    got_k = c.dk.double().cpu().numpy()
    assert np.all(np.abs(got_k - want_k) <= append_tolerance(dtype, want_k))
    assert np.array_equal(got_k[~c.used], c.k[~c.used])
    got_q = q_out.double().cpu().numpy()
    assert np.all(np.abs(got_q[:c.n] - want_q[:c.n]) <= append_tolerance(dtype, want_q[:c.n]))
    assert np.all(got_q[c.n:] == 7.0)


def test_append_without_queries_and_in_place(gto):
    c = dc.Case([3, 4], [10, 20], 4, 2, 64, 16, "bf16", seed=5, poison=0.0)
    f = torch.tensor(10000.0 ** (-np.arange(32) / 32), device=DEV)
    k, v = c.tensor(c.rng.normal(size=(c.T, 2, 64))), c.tensor(c.rng.normal(size=(c.T, 2, 64)))
    ctx = c.ctx(gto)
    k2, v2 = c.dk.clone(), c.dv.clone()
    q_out = torch.zeros_like(c.dq)
    gto.gto_kv_append(ctx, c.batch, c.dq, k, v, q_out, c.dk, c.dv, f)
    gto.gto_kv_append(ctx, c.batch, None, k, v, None, k2, v2, f)
    assert torch.equal(k2, c.dk) and torch.equal(v2, c.dv)
    q = c.dq.clone()
    gto.gto_kv_append(ctx, c.batch, q, k, v, q, k2, v2, f)
    assert torch.equal(q[:c.n], q_out[:c.n]) and torch.equal(q[c.n:], c.dq[c.n:])


# ------------------------------------------------------------------ gto_tree_attention

def check_attention(gto, c, scale=None, lse=True, stream=None, ctx=None):
    scale = c.dh ** -0.5 if scale is None else scale
    ctx = ctx or c.ctx(gto, softmax_scale=scale)
    out = torch.full((c.T, c.hq, c.dh), 5.0, dtype=c.dq.dtype, device=c.device)
    z = torch.full((c.T, c.hq), 5.0, device=c.device) if lse else None
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z, stream=stream)
    torch.cuda.synchronize(c.device)
    assert gto.gto_decode_status(ctx) == 0
    compare_attention(c, scale, out, z)


def compare_attention(c, scale, out, z, want=None):
    want, want_z, spread = want or dec.attention(c.host, c.q, c.k, c.v, c.page, scale, c.g)
    # a score is a sum of dh products in fp32, in any order: off by at most (dh + 2) 2^-23 sum |q k| scale (a tensor
    # core may cut instead of round, hence 2^-23), plus 2^-22 |score| for the exponential's argument; exp then errs by
    # twice that relative to itself in numerator and denominator.  A weight rounded to the type and the result rounded
    # once add half a step each of sum p |v| and |out|.
    x_abs = scale * np.abs(np.nan_to_num(c.k[c.used])).max() * np.abs(c.q).max() * c.dh ** 0.5 * 2 * c.dh ** 0.5
    ds = x_abs * (c.dh + 4) * 2.0 ** -23
    half = dc.HALF_STEP[c.dtype]
    n = c.n
    got = out.double().cpu().numpy()
    if n:
        tol = spread[:n] * (2 * ds + half + 2.0 ** -20) + half * np.abs(want[:n]) + 1e-30
        err = np.abs(got[:n] - want[:n])
        assert np.all(err <= tol), (np.max(err / tol), np.unravel_index(np.argmax(err / tol), err.shape))
    assert np.all(got[n:] == 5.0)                      # rows of no sequence
    if z is not None:
        got_z = z.double().cpu().numpy()
        empty = np.isneginf(want_z[:n])
        assert np.array_equal(np.isneginf(got_z[:n]), empty)
        if n:
            err = np.abs(got_z[:n][~empty] - want_z[:n][~empty])
            assert np.all(err <= 2 * ds + 2.0 ** -21 * (1 + np.abs(want_z[:n][~empty])))
        assert np.all(got_z[n:] == 5.0)


SHAPES = [(4, 2, 64), (8, 8, 128), (8, 1, 128), (10, 2, 64), (3, 3, 80), (2, 1, 256)]
LENS = [
    ([1], [1]),                                      # one token, nothing before it
    ([1, 1, 1, 1], [1, 127, 128, 129]),              # around a tile
    ([1, 1], [777, 64]),
    ([5, 0, 1, 17], [5, 3, 200, 17]),                # a prompt, no chunk, a prompt that fills the cache
    ([40, 130], [300, 131]),                         # more rows than one block
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("lens", range(len(LENS)))
def test_attention_causal(gto, lens, shape, dtype):
    hq, hkv, dh = shape
    q_lens, kv_lens = LENS[lens]
    page = [16, 8, 64, 32, 128][(lens + hq) % 5]
    c = dc.Case(q_lens, kv_lens, hq, hkv, dh, page, dtype, seed=lens, head_major=lens % 2 == 1)
    check_attention(gto, c)


TREES = [
    # q_lens, kv_lens, g, D, n_nodes
    ([13], [13], 12, 3, None),                       # nothing cached
    ([13, 12, 20], [140, 128, 256], 12, 3, None),    # lead 1, 0, 8; the tree across a tile's end
    ([61, 62], [61, 190], 60, 7, None),
    ([101], [229], 100, 8, None),                    # two mask words, the tree across two tiles
    ([129, 128], [300, 128], 128, 16, None),         # the largest tree
    ([7, 3, 0, 31], [90, 50, 40, 31], 30, 5, [5, 0, 0, 30]),   # ragged trees, a plain chunk among them
]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", [(4, 2, 64), (8, 1, 128), (4, 4, 128), (6, 2, 48)])
@pytest.mark.parametrize("tree", range(len(TREES)))
def test_attention_trees(gto, tree, shape, dtype):
    hq, hkv, dh = shape
    q_lens, kv_lens, g, D, n_nodes = TREES[tree]
    page = [16, 64, 8, 128][(tree + hq) % 4]
    c = dc.Case(q_lens, kv_lens, hq, hkv, dh, page, dtype, g, D, n_nodes, seed=tree + 50, head_major=tree % 2 == 0)
    check_attention(gto, c, lse=tree != 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_rows_whose_mask_is_empty(gto, dtype):
    c = dc.Case([6, 9], [6, 9], 4, 2, 64, 16, dtype, 6, 3, [6, 6], seed=9)
    c.host["node_mask"][0, 2:4] = False              # sequence 0 has no cache and no lead: these rows see nothing
    c.host["node_mask"][1, 0] = False                # sequence 1 has a lead of 3
    c.batch["node_mask"] = torch.from_numpy(dc.words(c.host["node_mask"])).to(DEV)
    check_attention(gto, c)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_attention_ignores_what_a_row_does_not_see(gto, dtype, bad):
    """Keys and values of one branch hold NaN or inf: only rows that see them change."""
    c = dc.Case([13], [70], 4, 2, 64, 16, dtype, 12, 3, seed=11)
    node = 5
    page, place = dec.slots(c.host, 0, [70 - 12 + node], c.page)
    blind = [0] + [1 + n for n in range(12) if not c.host["node_mask"][0, n, node]]
    c.k[page, place] = bad
    c.v[page, place] = bad
    c.dk, c.dv = c.pool(c.k), c.pool(c.v)
    ctx = c.ctx(gto)
    out = torch.zeros((c.T, c.hq, c.dh), dtype=c.dq.dtype, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out)
    good = dc.Case([13], [70], 4, 2, 64, 16, dtype, 12, 3, seed=11)
    want, _, spread = dec.attention(good.host, good.q, good.k, good.v, good.page, 0.125, 12)
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got[blind] - want[blind]) <= spread[blind] * (dc.HALF_STEP[dtype] * 2 + 1e-3))
    assert np.isnan(got[1 + node]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores(gto, dtype):
    """Scores of several hundred that rise and fall along the cache: the running maximum moves often."""
    c = dc.Case([3], [700], 4, 2, 128, 16, dtype, seed=12, scale=6.0)
    check_attention(gto, c, scale=0.25)


def test_attention_reads_queries_out_of_a_projection(gto):
    c = dc.Case([3, 2], [30, 90], 4, 2, 64, 16, "bf16", seed=13)
    qkv = torch.full((c.T, 8, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    qkv[:, :4] = c.dq
    ctx = c.ctx(gto)
    a, b = torch.zeros_like(c.dq), torch.zeros_like(c.dq)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, a)
    gto.gto_tree_attention(ctx, c.batch, qkv[:, :4], c.dk, c.dv, b)
    assert torch.equal(a, b)


LONG = [
    # sequences, tokens, longest cache, g, D: enough entries that every SM goes through several blocks of many tiles
    (96, 1, 3000, 0, 1), (24, 61, 2500, 60, 7), (3, 900, 4000, 0, 1), (40, 2, 4500, 0, 1), (7, 130, 6000, 128, 9),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(8, 8, 64), (16, 4, 128)])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_attention_long_batches(gto, case, shape, dtype):
    """Ragged lengths; the result does not change from call to call, bit for bit."""
    S, n, L, g, D = LONG[case]
    hq, hkv, dh = shape
    rng = np.random.default_rng(case)
    q_lens = [n if g else int(rng.integers(1, n + 1)) for _ in range(S)]
    kv_lens = [q + int(rng.integers(0, L)) for q in q_lens]
    c = dc.Case(q_lens, kv_lens, hq, hkv, dh, [16, 64, 128, 8, 32][case], dtype, g, D, seed=case, scale=1.2)
    ctx = c.ctx(gto)
    out = torch.full((c.T, hq, dh), 5.0, dtype=c.dq.dtype, device=DEV)
    z = torch.full((c.T, hq), 5.0, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
    again, z2 = torch.full_like(out, 5.0), torch.full_like(z, 5.0)
    for _ in range(3):
        gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, again, lse=z2)
    assert gto.gto_decode_status(ctx) == 0
    assert torch.equal(out, again) and torch.equal(z, z2)
    compare_attention(c, dh ** -0.5, out, z, c.attention_on_device(dh ** -0.5))


# ------------------------------------------------------------------ gto_verify_tree

def verify_case(rng, S, g, D, V, Vd, dtype, n_nodes=None, spread=1.5):
    trees = [dc.random_tree(rng, g, D) for _ in range(S)]
    parent = np.stack([t[0] for t in trees]) if g else np.zeros((S, 0), np.int32)
    token = rng.integers(0, Vd, size=(S, g)).astype(np.int32)
    d2t = None if V == Vd else rng.permutation(V)[:Vd].astype(np.int32)
    z = rng.normal(size=(S, 1 + g, V)) * spread
    for s in range(S):
        for n in range(g):
            x = token[s, n] if d2t is None else d2t[token[s, n]]
            z[s, 1 + parent[s, n], x] += rng.uniform(0, 1.0) + np.log(V)
    return dict(parent=parent, token=token, d2t=d2t, target=dc.round_to(z, dtype), u_node=rng.random((S, g)).astype(np.float32),
                u_bonus=rng.random(S).astype(np.float32), n_nodes=n_nodes,
                temperature=np.where(np.arange(S) % 3 == 2, 0.0, rng.uniform(0.3, 1.5, S)).astype(np.float32))


def run_verify(gto, c, D, V, Vd, dtype, ctx=None):
    S, g = c["parent"].shape
    cfg = gto.make_decode_config(S=S, g=g, D=D, V_draft=Vd, V_target=V, logit_dtype=dtype)
    ctx = ctx or gto.gto_decode_create(cfg, 0)
    out = gto.alloc_verdict(cfg, DEV)
    for t in out.values():
        t.fill_(-77)
    t = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)
    tree = dict(node_token=t(c["token"]), node_parent=t(c["parent"]))
    if c["n_nodes"] is not None:
        tree["n_nodes"] = t(np.array(c["n_nodes"], np.int32))
    target = t(c["target"]).to(dc.TORCH[dtype])
    gto.gto_verify_tree(ctx, tree, target, t(c["d2t"]), t(c["temperature"]), t(c["u_node"]), t(c["u_bonus"]), out)
    return ctx, {k: v.cpu().numpy() for k, v in out.items()}


def check_verdict(c, s, out, D):
    g = c["parent"].shape[1] if c["n_nodes"] is None else c["n_nodes"][s]
    path, ids, last, margin = dec.verify(c["parent"][s][:g], c["token"][s][:g], 1 + np.arange(g), c["target"][s],
                                         float(c["temperature"][s]), c["u_node"][s].astype(float), float(c["u_bonus"][s]), D, c["d2t"])
    assert margin > 1e-13            # the inputs put no decision where two fp64 orders of summation could differ
    assert out["accept_len"][s] == len(path)
    assert list(out["path_node"][s]) == path + [-1] * (D - len(path))
    assert list(out["token"][s]) == ids + [last] + [-1] * (D - len(path))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("S,g,D,V,Vd", [
    (5, 12, 3, 512, 512), (33, 60, 7, 1000, 200), (3, 1, 1, 16, 16), (4, 0, 1, 2048, 2048), (6, 128, 16, 4104, 4104),
    (2, 40, 5, 32000, 8000)])
def test_verify(gto, S, g, D, V, Vd, dtype):
    if V * (4 if dtype == "f32" else 2) % 16:
        V += 8
    c = verify_case(np.random.default_rng(S + V), S, g, D, V, Vd if Vd < 500 or Vd != V else V, dtype)
    Vd = V if c["d2t"] is None else len(c["d2t"])
    ctx, out = run_verify(gto, c, D, V, Vd, dtype)
    assert gto.gto_decode_status(ctx) == 0
    for s in range(S):
        check_verdict(c, s, out, D)


def test_verify_ragged_trees_masked_tokens_and_repeated_siblings(gto):
    rng = np.random.default_rng(1)
    c = verify_case(rng, 12, 10, 4, 256, 256, "f32", n_nodes=[0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 10])
    c["target"][rng.random(c["target"].shape) < 0.5] = -np.inf       # a grammar's mask
    c["target"][:, :, 0] = 0.0
    c["target"][11, :, 128:] = torch.finfo(torch.float32).min         # masked with the lowest value
    c["token"][:, 1] = c["token"][:, 0]
    c["parent"][:, :2] = -1
    _, out = run_verify(gto, c, 4, 256, 256, "f32")
    for s in range(12):
        check_verdict(c, s, out, 4)


def test_verify_uniforms_at_their_ends(gto):
    c = verify_case(np.random.default_rng(2), 8, 12, 3, 512, 512, "f32")
    c["u_node"][:4] = 0.0                                             # every first child is accepted
    c["u_node"][4:] = np.float32(1 - 2.0 ** -24)
    c["u_bonus"][::2], c["u_bonus"][1::2] = 0.0, np.float32(1 - 2.0 ** -24)
    c["temperature"][:] = 1.0
    _, out = run_verify(gto, c, 3, 512, 512, "f32")
    for s in range(8):
        path, ids, last, _ = dec.verify(c["parent"][s], c["token"][s], 1 + np.arange(12), c["target"][s], 1.0,
                                        c["u_node"][s].astype(float), float(c["u_bonus"][s]), 3)
        assert list(out["path_node"][s]) == path + [-1] * (3 - len(path))
        assert out["token"][s, len(path)] == last


@pytest.mark.parametrize("temperature", [1.0, 1e-3, 1e-30, 300.0])
@pytest.mark.parametrize("S,V", [(3, 32000), (70, 4096)])
def test_verify_flat_rows(gto, S, V, temperature):
    """Rows whose tokens all weigh about the same: every border is nearer than fp32 sums can tell."""
    rng = np.random.default_rng(V + S)
    c = verify_case(rng, S, 6, 3, V, V, "f32")
    c["target"] = np.round(rng.normal(size=c["target"].shape) * 0.05, 3)
    c["target"] = dc.round_to(c["target"], "f32")
    c["temperature"][:] = temperature
    c["u_node"][:] = rng.random((S, 6)).astype(np.float32) * np.float32(3.0 / V)   # next to the children's probabilities
    ctx, out = run_verify(gto, c, 3, V, V, "f32")
    assert gto.gto_decode_status(ctx) == 0
    for s in range(S):
        path, ids, last, margin = dec.verify(c["parent"][s], c["token"][s], 1 + np.arange(6), c["target"][s], float(c["temperature"][s]),
                                             c["u_node"][s].astype(float), float(c["u_bonus"][s]), 3)
        if margin > 1e-13:
            assert list(out["path_node"][s]) == path + [-1] * (3 - len(path))
            assert list(out["token"][s]) == ids + [last] + [-1] * (3 - len(path))


def test_verify_reports_rows_that_hold_no_distribution(gto):
    """NaN, +inf or nothing at all in a visited row; a bad temperature: reported, the sequence ends there."""
    c = verify_case(np.random.default_rng(3), 6, 12, 3, 512, 512, "f32")
    c["temperature"][:] = [1, 1, 1, 0, -1, 1]
    c["target"][0, 0, 7] = np.nan
    c["target"][1, 0, 9] = np.inf
    c["target"][2, 0, :] = -np.inf
    c["target"][3, 0, 500] = np.nan
    ctx, out = run_verify(gto, c, 3, 512, 512, "f32")
    assert gto.gto_decode_status(ctx) == 5
    assert gto.gto_decode_status(ctx) == 0                            # read and cleared
    assert np.all(out["accept_len"][:5] == 0) and np.all(out["token"][:5] == -1) and np.all(out["path_node"][:5] == -1)
    check_verdict(c, 5, out, 3)


def test_verify_reports_indices_out_of_range(gto):
    c = verify_case(np.random.default_rng(4), 5, 6, 3, 512, 512, "f32", n_nodes=[6, 6, 6, 9, 6])
    c["token"][0, 0], c["token"][1, 1] = 512, -1
    c["parent"][2, 3] = 4                                             # a parent after its child
    ctx, out = run_verify(gto, c, 3, 512, 512, "f32")
    assert gto.gto_decode_status(ctx) == 8
    c["n_nodes"] = [6] * 5
    check_verdict(c, 4, out, 3)
    assert out["accept_len"][3] == 0


def test_verify_in_the_layout_of_the_reward_pass(gto):
    """The training pass's trees and target rows: the greedy walk is its longest accepted sequence, and the mean of
    accept_len over many draws at temperature 1 is its expected number of accepted tokens (5 sigma)."""
    import harness
    w = synth.Workload("t", B=16, V_draft=512, V_target=2048, D=4, k=4, g=20, dtype="f32", seed=8, sigma_t=1.0, boost=8.0)
    p, data = harness.run_pass(w, DEV)
    S, N = w.B, 400
    cfg = gto.make_decode_config(S=S * N, g=w.g, D=w.D, k=w.k, V_draft=w.V_draft, V_target=w.V_target, logit_dtype=w.dtype,
                                 flags=gto.GTO_DECODE_CONTEXT_ROWS)
    ctx = gto.gto_decode_create(cfg, 0)
    names = ("node_token", "node_parent", "node_depth", "node_slot")
    tree = {n: p.tree[n][0].contiguous() for n in names}
    target = data["target"][0].contiguous()
    out = gto.alloc_verdict(cfg, DEV, S)
    zero = torch.zeros(S, device=DEV)
    gto.gto_verify_tree(ctx, tree, target, data["d2t"], zero, torch.zeros(S, w.g, device=DEV), zero, out)
    assert torch.equal(out["accept_len"], p.reward["path_len"])
    assert torch.equal(out["path_node"], p.reward["path_node"])
    gen = torch.Generator(DEV).manual_seed(1)
    many = {n: tree[n].repeat(N, 1) for n in names}
    out = gto.alloc_verdict(cfg, DEV)
    gto.gto_verify_tree(ctx, many, target.repeat(N, 1, 1), data["d2t"], torch.ones(S * N, device=DEV),
                        torch.rand((S * N, w.g), generator=gen, device=DEV), torch.rand(S * N, generator=gen, device=DEV), out)
    assert gto.gto_decode_status(ctx) == 0
    got = out["accept_len"].view(N, S).double()
    want = p.reward["etree"][0]
    assert torch.all((got.mean(0) - want).abs() <= 5 * got.std(0) / N ** 0.5 + 1e-6)


# ------------------------------------------------------------------ gto_kv_commit

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layers", [1, 3])
def test_commit_moves_the_accepted_entries_and_nothing_else(gto, layers, dtype):
    g, D = 40, 12
    c = dc.Case([41, 40, 0, 7, 45], [60, 200, 9, 30, 45], 4, 2, 64, 16, dtype, g, D, [40, 40, 0, 5, 40], seed=3, poison=2.0)
    ctx = c.ctx(gto)
    rng = np.random.default_rng(4)
    length = np.array([12, 3, 0, 5, 0], np.int32)
    path = np.full((5, D), -1, np.int32)
    path[0] = np.sort(rng.choice(g, 12, replace=False))
    path[1, :3] = [0, 1, 39]
    path[3, :5] = np.arange(5)
    k = torch.stack([c.dk + i for i in range(layers)])
    v = torch.stack([c.dv - i for i in range(layers)])
    want_k, want_v = k.clone(), v.clone()
    for s, (q0, n, L, base, nodes, lead) in enumerate(dec.chunks(c.host, g)):
        for j in range(length[s]):
            p0, r0 = dec.slots(c.host, s, base + lead + path[s, j], 16)
            p1, r1 = dec.slots(c.host, s, base + lead + j, 16)
            want_k[:, int(p1), int(r1)] = k[:, int(p0), int(r0)]
            want_v[:, int(p1), int(r1)] = v[:, int(p0), int(r0)]
    verdict = dict(accept_len=torch.from_numpy(length).to(DEV), path_node=torch.from_numpy(path).to(DEV),
                   token=torch.zeros((5, D + 1), dtype=torch.int32, device=DEV))
    new_len = torch.full((5,), -5, dtype=torch.int32, device=DEV)
    if layers == 1:
        gto.gto_kv_commit(ctx, c.batch, verdict, k[0], v[0], new_len)
    else:
        gto.gto_kv_commit(ctx, c.batch, verdict, k, v, new_len)
    assert gto.gto_decode_status(ctx) == 0
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    assert new_len.tolist() == [20 + 12, 160 + 3, 9, 25 + 5, 5]


# ------------------------------------------------------------------ data faults

def test_inconsistent_batches_are_reported_and_skipped(gto):
    """Each table in turn; the other sequences' rows are right, the bad one's are left alone (page tables: unspecified)."""
    for what in ("q_start", "kv_len", "n_nodes", "page", "chunk's page"):
        c = dc.Case([7, 7, 7], [30, 40, 50], 4, 2, 64, 16, "f32", 6, 3, [6, 6, 6], seed=1)
        if what == "q_start":
            c.batch["q_start"][2] = 5000
        elif what == "kv_len":
            c.batch["kv_len"][1] = 6
        elif what == "n_nodes":
            c.batch["n_nodes"][1] = 7
        else:
            c.batch["page_table"][1, 0 if what == "page" else 2] = c.n_pages
        ctx = c.ctx(gto)
        out = torch.full((c.T, 4, 64), 5.0, device=DEV)
        gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out)
        assert gto.gto_decode_status(ctx) == 8, what
        want, _, spread = dec.attention(c.host, c.q, c.k, c.v, c.page, 0.125, 6)
        got = out.double().cpu().numpy()
        good = [r for s in ((0,) if what == "q_start" else (0, 2)) for r in range(7 * s, 7 * s + 7)]
        assert np.all(np.abs(got[good] - want[good]) <= spread[good] * 1e-4), what
        if what in ("kv_len", "n_nodes"):
            assert np.all(got[7:14] == 5.0), what
        k, v = c.tensor(c.rng.normal(size=(c.T, 2, 64))), c.tensor(c.rng.normal(size=(c.T, 2, 64)))
        f = torch.tensor(10000.0 ** (-np.arange(32) / 32), device=DEV)
        gto.gto_kv_append(ctx, c.batch, None, k, v, None, c.dk, c.dv, f)
        # the chunk's entries 33..39 are in the third page: the first is not followed
        assert gto.gto_decode_status(ctx) == (0 if what == "page" else 8), what


def test_commit_reports_a_path_that_does_not_increase(gto):
    c = dc.Case([7, 7], [30, 40], 4, 2, 64, 16, "f32", 6, 3, seed=1, poison=0.0)
    ctx = c.ctx(gto)
    k, v = c.dk.clone(), c.dv.clone()
    verdict = dict(accept_len=torch.tensor([2, 2], dtype=torch.int32, device=DEV),
                   path_node=torch.tensor([[3, 3, -1], [1, 6, -1]], dtype=torch.int32, device=DEV),
                   token=torch.zeros((2, 4), dtype=torch.int32, device=DEV))
    new_len = torch.full((2,), -5, dtype=torch.int32, device=DEV)
    gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, new_len)
    assert gto.gto_decode_status(ctx) == 8
    assert torch.equal(k, c.dk) and torch.equal(v, c.dv) and new_len.tolist() == [-5, -5]
