"""Sampling, verification under limits and the page calls together, as a decoding loop makes them: prompts forked into
continuations, drafted trees, pages given back and moved, against a plain fp64 model and the oracle."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import limits_oracle as lim
from oracle import pages_oracle as pg
from test_decode_step_gpu import Model

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# fp32 sums of a few hundred terms of size ~6 put the logits off by 1e-5: no decision is taken nearer to its border.
CLEAR = 1e-4


class Rows:
    """Target rows of a tree, found when they are looked at: row 0 follows the sequence, row 1 + n the path to node n."""

    def __init__(self, m, tokens, parent, token):
        self.m, self.tokens, self.parent, self.token = m, tokens, parent, token

    def __getitem__(self, row):
        path, n = [], row - 1
        while n >= 0:
            path.append(int(self.token[n]))
            n = int(self.parent[n])
        return self.m.logits(self.tokens + path[::-1])[-1]


def settings(rng, S):
    s = dict(temperature=rng.uniform(0.7, 1.3, S), top_k=rng.integers(3, 60, S), top_p=rng.uniform(0.6, 1.0, S), min_p=rng.uniform(0.0, 0.05, S))
    s["temperature"][1], s["top_k"][2], s["top_p"][3] = 0.0, 0, 1.0
    return {k: v.astype(np.int32 if k == "top_k" else np.float32) for k, v in s.items()}


@pytest.mark.parametrize("shape", [(4, 2, 64), (3, 1, 128)])
def test_continuations_of_two_prompts_are_the_plain_models(shape):
    from paper_2509_22134_b200 import binding as gto
    from paper_2509_22134_b200.runner import DecodeStep
    m = Model(256, *shape, layers=2, seed=50 + shape[0])
    rng = np.random.default_rng(shape[0])
    S, g, D, page = 6, 10, 4, 8
    cfg = gto.make_decode_config(S=S, T=S * 40, n_q_heads=m.hq, n_kv_heads=m.hkv, head_dim=m.dh, page_size=page, n_pages=80, max_pages=14,
                                 dtype="f32", g=g, D=D, V_draft=m.V, V_target=m.V, logit_dtype="f32", flags=gto.GTO_DECODE_PAGES)
    step = DecodeStep(cfg, m.layers, m.inv_freq, DEV)
    on = lambda x: torch.tensor(np.asarray(x), dtype=torch.float32, device=DEV)
    ints = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)
    emb, w_in, w_out, w_end = on(m.emb), on(m.w_in), on(m.w_out), on(m.w_end)

    def forward(tokens):
        x = emb[torch.tensor(tokens, device=DEV)]
        for i in range(m.layers):
            y = (x @ w_in[i]).view(len(tokens), -1, m.dh)
            out = torch.zeros((len(tokens), m.hq, m.dh), device=DEV)
            step.attend(i, y[:, :m.hq], y[:, m.hq:m.hq + m.hkv], y[:, m.hq + m.hkv:], out)
            x = x + out.reshape(len(tokens), -1) @ w_out[i]
            x = x / x.square().mean(-1, keepdim=True).sqrt()
        return x @ w_end

    def keeps_its_rules():
        pg.check({k: v.cpu().numpy() for k, v in step.pool.items()}, page)
        assert step.status() == 0

    s = settings(rng, S)
    limits = {k: torch.from_numpy(s[k]).to(DEV) for k in ("top_k", "top_p", "min_p")}
    heat = torch.from_numpy(s["temperature"]).to(DEV)
    one = lambda i: {k: (int if k == "top_k" else float)(v[i]) for k, v in s.items()}
    # ---- the prompts, in sequences 0 and 3
    prompts = {0: rng.integers(0, m.V, 21).tolist(), 3: rng.integers(0, m.V, 16).tolist()}
    lens = np.array([len(prompts.get(i, [])) for i in range(S)])
    step.reserve(ints(lens))
    start = np.concatenate([[0], np.cumsum(lens)])
    step.begin(ints(start))
    logits = forward(sum((prompts.get(i, []) for i in range(S)), []))
    step.commit()
    assert step.kv_len.tolist() == lens.tolist()
    # ---- three continuations each, whose first tokens are drawn from two rows
    parent = np.array([0, 0, 0, 3, 3, 3])
    step.fork(ints(parent))
    keeps_its_rules()
    tokens = [list(prompts[int(parent[i])]) for i in range(S)]
    rows = start[parent + 1] - 1
    want, u = [], np.zeros(S, np.float32)
    for i in range(S):
        z, margin = m.logits(tokens[i])[-1], 0.0
        while margin < CLEAR:
            u[i] = rng.random(dtype=np.float32)
            token, logp, n, margin = lim.sample(z, u=float(u[i]), **one(i))
        want.append((token, logp, n))
    drawn = step.sample(logits, heat, torch.from_numpy(u).to(DEV), limits, rows=ints(rows))
    assert drawn["token"].tolist() == [w[0] for w in want] and drawn["n_kept"].tolist() == [w[2] for w in want]
    assert np.abs(drawn["logp"].cpu().numpy() - [w[1] for w in want]).max() < CLEAR
    for i in range(S):
        tokens[i].append(want[i][0])
    # ---- steps with drafted trees
    accepted = 0
    for turn in range(5):
        nodes = rng.integers(0, g + 1, S).astype(np.int32)
        trees = [dc.random_tree(rng, g, D) for _ in range(S)]
        token = rng.integers(0, m.V, (S, g)).astype(np.int32)
        for i in range(S):                 # half of the nodes are what the model finds likely there
            rows_i = Rows(m, tokens[i], trees[i][0], token[i])
            for n in range(nodes[i]):
                if rng.random() < 0.5:
                    token[i, n] = np.argsort(-rows_i[int(trees[i][0][n]) + 1])[rng.integers(0, 3)]
        tree = dict(node_token=torch.from_numpy(token), node_parent=torch.from_numpy(np.stack([t[0] for t in trees])),
                    node_depth=torch.from_numpy(np.stack([t[1] for t in trees])),
                    node_mask=torch.from_numpy(dc.words(np.stack([t[2] for t in trees]))), n_nodes=torch.from_numpy(nodes))
        tree = {n: x.to(DEV) for n, x in tree.items()}
        chunk = [[tokens[i][-1]] + token[i, :nodes[i]].tolist() for i in range(S)]
        start = np.concatenate([[0], np.cumsum([len(c) for c in chunk])])
        step.reserve(step.kv_len + ints([len(c) for c in chunk]))
        keeps_its_rules()
        if turn == 0:                      # the continuations write into pages of their own, and share the full ones
            table = step.page_table.cpu().numpy()
            assert (table[0, :2] == table[1, :2]).all() and len({int(table[i, 2]) for i in range(3)}) == 3
        step.begin(ints(start), tree)
        logits = forward(sum(chunk, []))
        target = torch.zeros((S, 1 + g, m.V), device=DEV)
        for i in range(S):
            target[i, :len(chunk[i])] = logits[start[i]:start[i + 1]]
        u_node, u_bonus, answer = np.zeros((S, g), np.float32), np.zeros(S, np.float32), []
        for i in range(S):
            margin, k = 0.0, int(nodes[i])
            while margin < CLEAR:
                u_node[i], u_bonus[i] = rng.random(g, dtype=np.float32), rng.random(dtype=np.float32)
                path, ids, last, margin = lim.verify(trees[i][0][:k], token[i][:k], 1 + np.arange(k), Rows(m, tokens[i], trees[i][0], token[i]),
                                                     u_node=u_node[i].astype(float), u_bonus=float(u_bonus[i]), D=D, **one(i))
            answer.append((path, ids, last))
        verdict = step.verify(tree, target, None, heat, torch.from_numpy(u_node).to(DEV), torch.from_numpy(u_bonus).to(DEV), limits)
        step.commit()
        for i, (path, ids, last) in enumerate(answer):
            assert verdict["accept_len"][i].item() == len(path)
            assert verdict["token"][i].tolist() == ids + [last] + [-1] * (D - len(ids))
            tokens[i] += ids + [last]
            accepted += len(ids)
        assert step.kv_len.tolist() == [len(t) - 1 for t in tokens]
        step.reserve(step.kv_len.clone())  # what was not accepted goes back
        keeps_its_rules()
        assert step.pool["held"].tolist() == [-(-(len(t) - 1) // page) for t in tokens]
        if turn % 2 == 0:
            used = int(step.compact())
            keeps_its_rules()
            assert int((step.pool["ref_count"][:used] > 0).sum()) == used == int((step.pool["ref_count"] > 0).sum())
        if turn == 2:                      # sequence 4 ends, and a second copy of 2 takes its place
            step.fork(ints([0, 1, 2, 3, 2, 5]))
            tokens[4] = list(tokens[2])
            keeps_its_rules()
    assert accepted > 0
    step.fork(ints([-1] * S))
    assert not step.pool["ref_count"].any() and not step.kv_len.any()
    step.close()


def test_a_step_without_limits_or_pages_is_as_before():
    from paper_2509_22134_b200 import binding as gto
    from paper_2509_22134_b200.runner import DecodeStep
    cfg = gto.make_decode_config(S=2, T=8, n_q_heads=2, n_kv_heads=1, head_dim=64, page_size=8, n_pages=4, max_pages=2, V_draft=64, V_target=64)
    step = DecodeStep(cfg, 1, np.ones(32), DEV)
    assert step.pool is None
    z = torch.zeros((2, 64), dtype=torch.bfloat16, device=DEV)
    z[0, 5] = z[1, 9] = 4.0
    out = step.sample(z, torch.zeros(2, device=DEV), torch.zeros(2, device=DEV))
    assert out["token"].tolist() == [5, 9] and out["logp"].tolist() == [0, 0] and out["n_kept"].tolist() == [1, 1]
    with pytest.raises(ValueError):
        step.fork(torch.zeros(2, dtype=torch.int32, device=DEV))
    step.close()
