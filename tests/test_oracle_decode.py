"""Pins of the decoding-step oracle: rotations against complex multiplication and the relative-position
property, attention against torch in fp64, verification against the target's distribution and against
the tree reward's expected number of accepted tokens."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as dec
from oracle import gto_oracle as orc


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product_and_scores_depend_on_distance_only(interleaved):
    rng = np.random.default_rng(0)
    f = 10000.0 ** (-np.arange(8) / 8)
    x, y = rng.normal(size=20), rng.normal(size=20)
    got = dec.rotate(x, 77, f, interleaved)
    z = x[:16].reshape(8, 2) if interleaved else x[:16].reshape(2, 8).T
    w = (z[:, 0] + 1j * z[:, 1]) * np.exp(1j * 77 * f)
    want = np.stack([w.real, w.imag], 1)
    want = want.reshape(-1) if interleaved else want.T.reshape(-1)
    assert np.allclose(got[:16], want, atol=1e-14) and np.array_equal(got[16:], x[16:])
    a = dec.rotate(x, 905, f, interleaved) @ dec.rotate(y, 900, f, interleaved)
    b = dec.rotate(x, 5, f, interleaved) @ dec.rotate(y, 0, f, interleaved)
    assert a == pytest.approx(b, abs=1e-10)


def test_norm_scales_to_unit_mean_square():
    x = np.random.default_rng(1).normal(size=(3, 32)) * 7
    y = dec.rotate(x, 0, np.zeros(0), weight=np.ones(32), eps=0.0)
    assert np.allclose((y * y).mean(1), 1.0)


def test_attention_matches_torch_in_64_bits_for_a_causal_chunk():
    rng = np.random.default_rng(2)
    n, L, hq, hkv, dh, page = 5, 19, 4, 2, 16, 4
    k, v = rng.normal(size=(6, page, hkv, dh)), rng.normal(size=(6, page, hkv, dh))
    q = rng.normal(size=(n, hq, dh))
    table = np.array([[3, 0, 5, 1, 2]])
    batch = dict(q_start=[0, n], kv_len=[L], page_table=table)
    out, lse, _ = dec.attention(batch, q, k, v, page, 0.3)
    flat = [torch.tensor(c[table[0]].reshape(-1, hkv, dh)[:L]).repeat_interleave(hq // hkv, 1).permute(1, 0, 2) for c in (k, v)]
    mask = torch.ones(n, L, dtype=torch.bool).tril(L - n)
    want = torch.nn.functional.scaled_dot_product_attention(torch.tensor(q).permute(1, 0, 2), flat[0], flat[1], attn_mask=mask, scale=0.3)
    assert np.allclose(out, want.permute(1, 0, 2).numpy(), atol=1e-12)
    x = (torch.tensor(q).permute(1, 0, 2) @ flat[0].transpose(1, 2) * 0.3).masked_fill(~mask, -np.inf)
    assert np.allclose(lse, torch.logsumexp(x, 2).T.numpy(), atol=1e-12)


def test_a_tree_row_equals_the_chain_of_its_ancestors():
    """Attention of a node under the mask = causal attention of the sequence that ends in it."""
    rng = np.random.default_rng(3)
    parent = [-1, -1, 0, 2, 1]
    g, base, dh, page = 5, 7, 16, 4
    L = base + 1 + g
    k, v = rng.normal(size=(4, page, 1, dh)), rng.normal(size=(4, page, 1, dh))
    q = rng.normal(size=(1 + g, 1, dh))
    mask = np.eye(g, dtype=bool)
    for n in range(g):
        if parent[n] >= 0:
            mask[n] |= mask[parent[n]]
    tree = dict(q_start=[0, 1 + g], kv_len=[L], page_table=[[0, 1, 2, 3]], node_mask=mask[None])
    out, lse, _ = dec.attention(tree, q, k, v, page, 0.25, g)
    flat_k, flat_v = k.reshape(-1, 1, dh), v.reshape(-1, 1, dh)
    for n in range(g):
        chain = list(np.nonzero(mask[n])[0])
        keep = list(range(base + 1)) + [base + 1 + a for a in chain]
        kk, vv = np.zeros((4 * page, 1, dh)), np.zeros((4 * page, 1, dh))
        kk[:len(keep)], vv[:len(keep)] = flat_k[keep], flat_v[keep]
        one = dict(q_start=[0, 1], kv_len=[len(keep)], page_table=[[0, 1, 2, 3]])
        o1, l1, _ = dec.attention(one, q[1 + n:2 + n], kk.reshape(4, page, 1, dh), vv.reshape(4, page, 1, dh), page, 0.25)
        assert np.allclose(o1[0], out[1 + n], atol=1e-13) and l1[0, 0] == pytest.approx(lse[1 + n, 0])


def test_verified_tokens_follow_the_target_distribution():
    """First emitted token over many uniforms: the target's law, with and without children (5 sigma)."""
    rng = np.random.default_rng(4)
    V, N = 7, 20000
    z = rng.normal(size=(3, V)) * 1.5
    p = np.exp(z[0] / 0.8) / np.exp(z[0] / 0.8).sum()
    for parent, token in (([], []), ([-1, -1], [2, 5]), ([-1, -1, -1], [1, 1, 0])):
        rows = [-1] * len(parent)
        count = np.zeros(V)
        for _ in range(N):
            path, ids, last, _ = dec.verify(parent, token, rows, z, 0.8, rng.random(len(parent)), rng.random(), 3)
            count[ids[0] if ids else last] += 1
        assert np.all(np.abs(count / N - p) < 5 * np.sqrt(p * (1 - p) / N) + 1e-12)


def test_mean_accepted_length_is_the_reward_passes_expected_number_of_accepted_tokens():
    """etree of the tree reward (sum of path products) is the mean of accept_len at temperature 1 (5 sigma)."""
    rng = np.random.default_rng(5)
    D, k, g, V, N = 3, 3, 9, 40, 4000
    draft = rng.normal(size=(D, k, V)) * 2.0
    target = rng.normal(size=(1 + (D - 1) * k, V)) * 1.0
    target[0] += draft[0, 0]
    target[1:] += draft[1:].reshape(-1, V)
    tree = orc.build_tree(draft, D, k, g)
    p, _ = orc.target_node_probs(tree, target)
    etree = orc.tree_reward(tree, p)["etree"]
    rows = [1 + (int(tree.depth[n]) - 1) * k + int(tree.slot[n]) if tree.slot[n] >= 0 and tree.depth[n] < D else -1
            for n in range(g)]
    got = [len(dec.verify(tree.parent, tree.token, rows, target, 1.0, rng.random(g), rng.random(), D)[0]) for _ in range(N)]
    assert abs(np.mean(got) - etree) < 5 * np.std(got) / np.sqrt(N)


def test_greedy_walk_is_the_reward_passes_longest_accepted_sequence():
    rng = np.random.default_rng(6)
    D, k, g, V = 4, 3, 14, 30
    for _ in range(20):
        draft = rng.normal(size=(D, k, V)) * 2.0
        target = np.concatenate([draft[0, :1], draft[1:].reshape(-1, V)]) + rng.normal(size=(1 + (D - 1) * k, V)) * 0.5
        tree = orc.build_tree(draft, D, k, g)
        rows = [1 + (int(tree.depth[n]) - 1) * k + int(tree.slot[n]) if tree.slot[n] >= 0 and tree.depth[n] < D else -1
                for n in range(g)]
        path, ids, last, _ = dec.verify(tree.parent, tree.token, rows, target, 0.0, np.zeros(g), 0.0, D)
        want = orc.longest_accepted(tree, target)
        assert path == [int(n) for n in want["nodes"]]
