"""The bounds of decode_bounds: what they let pass and what they do not (CPU), and the attention under them (GPU)."""
import numpy as np
import pytest
import torch

import decode_bounds as db
import decode_cases as dc

# q_lens, kv_lens, g, D, n_nodes, scale of queries and keys, softmax scale over dh^-1/2
BATCHES = {
    "prompts": ([5, 0, 1, 40], [5, 3, 200, 300], 0, 1, None, 1.0, 1.0),
    "trees": ([13, 7, 0, 31], [140, 50, 40, 31], 30, 5, [12, 5, 0, 30], 1.0, 1.0),
    "large scores": ([3, 1], [700, 130], 0, 1, None, 6.0, 2.0),
    "long": ([2, 1], [4500, 2900], 0, 1, None, 1.2, 1.0),
    "long trees": ([61, 30], [2500, 1200], 60, 7, [60, 29], 1.2, 1.0),
}


def batch(name, shape, dtype, device="cuda:0", page=16):
    q_lens, kv_lens, g, D, n_nodes, size, factor = BATCHES[name]
    c = dc.Case(q_lens, kv_lens, *shape, page, dtype, g, D, n_nodes, seed=len(name), device=device, poison=0.0, scale=size)
    return c, factor * shape[2] ** -0.5


def round_as(dtype):
    return lambda w: w.to(dc.TORCH[dtype]).double()


def computed(c, scale, **kw):
    """(out, lse) as a kernel would leave them."""
    r = db.expected(c, scale, **kw)
    return dc.round_to(r["out"], c.dtype), r["lse"].astype(np.float32).astype(np.float64)


SHAPE = (4, 2, 128)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("name", BATCHES)
def test_the_bounds_hold_a_right_result_and_no_wrong_one(name, dtype):
    c, scale = batch(name, SHAPE, dtype, "cpu")
    want = db.expected(c, scale)
    right = computed(c, scale, weights=None if dtype == "f32" else round_as(dtype))
    assert db.misses(want, *right) == []
    assert db.misses(want, np.zeros_like(right[0]), right[1])                    # nothing written
    assert db.misses(want, np.full_like(right[0], np.nan), right[1])
    assert db.misses(want, right[0], right[1] + 1e-3)
    if name == "large scores":                                                   # one entry has a row's weight: any will not do
        assert db.misses(want, *computed(c, scale, drop=lambda s, L: np.arange(L // 2)))
        return
    one, tile = (lambda s, L: [L // 3]), (lambda s, L: np.arange(L // 128 * 64, min(L, L // 128 * 64 + 64)) if s == 0 else [])
    for drop in (one, tile):                                                     # an entry of every row; a tile of one sequence
        assert db.misses(want, *computed(c, scale, drop=drop)), drop
    some = computed(c, scale, drop=one)
    row = c.n // 2
    mixed = right[0].copy(), right[1].copy()
    mixed[0][row, 0], mixed[1][row, 0] = some[0][row, 0], some[1][row, 0]        # an entry of one row of one head
    if np.abs(mixed[1] - right[1]).max() > 2e-5:                                 # (where it weighs anything)
        assert db.misses(want, *mixed)


@pytest.mark.parametrize("name", [n for n in BATCHES if n != "large scores"])    # (scores of 700 err by more than that in fp32)
def test_fp32_bounds_refuse_16_bit_arithmetic(name):
    c, scale = batch(name, SHAPE, "f32", "cpu")
    want = db.expected(c, scale)
    for coarse in ("bf16", "f16"):
        out, lse = computed(c, scale, dtype=coarse)                              # inputs
        assert any(m.startswith("out") for m in db.misses(want, out, lse)) and any(m.startswith("lse") for m in db.misses(want, out, lse))
        out, lse = computed(c, scale, weights=round_as(coarse))                  # weights
        assert any(m.startswith("out") for m in db.misses(want, out, lse))
        assert db.misses(want, dc.round_to(db.expected(c, scale)["out"], coarse), lse)      # results


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape,page", [((4, 2, 64), 16), ((8, 1, 128), 64), ((4, 4, 128), 8), ((10, 2, 64), 24), ((3, 3, 80), 16),
                                        ((2, 1, 256), 5), ((16, 2, 128), 128)])
@pytest.mark.parametrize("name", BATCHES)
def test_attention_within_the_bounds(name, shape, page, dtype):
    from paper_2509_22134_b200 import binding as gto
    c, scale = batch(name, shape, dtype, page=page)
    ctx = c.ctx(gto, softmax_scale=scale)
    out, lse = torch.zeros_like(c.dq), torch.zeros((c.T, c.hq), device="cuda:0")
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=lse)
    assert gto.gto_decode_status(ctx) == 0
    want = db.expected(c, scale, "cuda:0")
    assert db.misses(want, out.double().cpu().numpy()[:c.n], lse.double().cpu().numpy()[:c.n]) == []


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("S,n,L,g,hq,hkv,dh", [(96, 1, 3000, 0, 8, 8, 64), (24, 61, 2500, 60, 16, 4, 128), (3, 900, 4000, 0, 16, 4, 128),
                                               (7, 130, 6000, 128, 8, 8, 64), (300, 1, 200, 0, 8, 2, 128)])
def test_long_batches_within_the_bounds(S, n, L, g, hq, hkv, dh, dtype):
    """Work that is cut over all SMs and joined: a tile that a cut loses is outside the bounds."""
    from paper_2509_22134_b200 import binding as gto
    rng = np.random.default_rng(S)
    q_lens = [n if g else int(rng.integers(1, n + 1)) for _ in range(S)]
    c = dc.Case(q_lens, [q + int(rng.integers(0, L)) for q in q_lens], hq, hkv, dh, 32, dtype, g, 9, seed=S, scale=1.2, poison=0.0)
    scale = dh ** -0.5
    ctx = c.ctx(gto, softmax_scale=scale)
    out, lse = torch.zeros_like(c.dq), torch.zeros((c.T, c.hq), device="cuda:0")
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=lse)
    assert gto.gto_decode_status(ctx) == 0
    want = db.expected(c, scale, "cuda:0")
    assert db.misses(want, out.double().cpu().numpy()[:c.n], lse.double().cpu().numpy()[:c.n]) == []
