"""The decoding step's calls together, as a decoding loop makes them: against a plain fp64 model, against the oracle step
by step with the training pass's own trees, captured into graphs, on other streams, and at far addresses."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import decode_oracle as dec
from paper_2509_22134_b200 import synth
from test_decode_gpu import append_tolerance, compare_attention

DEV = "cuda:0"


# ------------------------------------------------------------------ a small model, plainly

class Model:
    """Attention layers with residual sums and a unit-mean-square norm after each, in fp64 on the CPU."""

    def __init__(self, V, hq, hkv, dh, layers, seed):
        rng = np.random.default_rng(seed)
        self.V, self.hq, self.hkv, self.dh, self.layers, self.E = V, hq, hkv, dh, layers, 64
        self.emb = rng.normal(size=(V, self.E))
        self.w_in = rng.normal(size=(layers, self.E, (hq + 2 * hkv) * dh)) / 8
        self.w_out = rng.normal(size=(layers, hq * dh, self.E)) / (hq * dh) ** 0.5
        self.w_end = rng.normal(size=(self.E, V)) * 0.75          # logits of a spread of about 6
        self.inv_freq = 10000.0 ** (-np.arange(dh // 2) / (dh // 2))

    def logits(self, tokens):
        """After every token of one sequence."""
        n = len(tokens)
        x = self.emb[tokens]
        angle = np.arange(n)[:, None] * self.inv_freq
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        turn = lambda y: np.concatenate([y[..., :self.dh // 2] * c - y[..., self.dh // 2:] * s,
                                         y[..., self.dh // 2:] * c + y[..., :self.dh // 2] * s], -1)
        for i in range(self.layers):
            y = (x @ self.w_in[i]).reshape(n, -1, self.dh)
            q, k, v = turn(y[:, :self.hq]), turn(y[:, self.hq:self.hq + self.hkv]), y[:, self.hq + self.hkv:]
            k, v = np.repeat(k, self.hq // self.hkv, 1), np.repeat(v, self.hq // self.hkv, 1)
            z = np.einsum("ihd,jhd->hij", q, k) * self.dh ** -0.5
            z = np.where(np.tril(np.ones((n, n), bool)), z, -np.inf)
            p = np.exp(z - z.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            x = x + np.einsum("hij,jhd->ihd", p, v).reshape(n, -1) @ self.w_out[i]
            x = x / np.sqrt(np.mean(x * x, -1, keepdims=True))
        return x @ self.w_end

    def greedy(self, tokens, n):
        """The n most likely tokens one after another, and how far the runner-up ever came."""
        tokens, margin = list(tokens), np.inf
        for _ in range(n):
            z = np.sort(self.logits(tokens)[-1])
            margin = min(margin, z[-1] - z[-2])
            tokens.append(int(np.argmax(self.logits(tokens)[-1])))
        return tokens[-n:], margin


MODELS = [(4, 2, 64), (3, 1, 128)]
PROMPTS = [7, 1, 30]
STEPS, LEVELS = 6, 4


def greedy_truth(shape):
    m = Model(256, *MODELS[shape], layers=2, seed=30 + shape)
    rng = np.random.default_rng(shape)
    prompts = [rng.integers(0, m.V, n).tolist() for n in PROMPTS]
    return m, prompts, [m.greedy(p, STEPS * (LEVELS + 1)) for p in prompts]


@pytest.mark.parametrize("shape", range(len(MODELS)))
def test_the_plain_models_greedy_tokens_are_clear(shape):
    """The next test compares tokens: its precondition.  fp32 sums of a few hundred terms of size ~6 err by 1e-5."""
    _, _, truth = greedy_truth(shape)
    assert min(margin for _, margin in truth) > 1e-3


def page_tables(rng, S, pages_each, max_pages):
    order = rng.permutation(S * pages_each).astype(np.int32).reshape(S, pages_each)
    table = np.full((S, max_pages), -1, np.int32)
    table[:, :pages_each] = order
    return torch.from_numpy(table)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", range(len(MODELS)))
def test_decoding_with_trees_gives_the_models_greedy_tokens(shape):
    """Drafts that are partly right, trees of other sizes in every step (and none), pages of 8: the tokens are the ones
    that the plain model finds one by one."""
    from paper_2509_22134_b200 import binding as gto
    from paper_2509_22134_b200.runner import DecodeStep
    m, prompts, truth = greedy_truth(shape)
    rng = np.random.default_rng(90 + shape)
    S, g, D, page = len(prompts), 12, LEVELS, 8
    cfg = gto.make_decode_config(S=S, T=S * 40, n_q_heads=m.hq, n_kv_heads=m.hkv, head_dim=m.dh, page_size=page, n_pages=S * 12,
                                 max_pages=13, dtype="f32", g=g, D=D, V_draft=m.V, V_target=m.V, logit_dtype="f32")
    step = DecodeStep(cfg, m.layers, m.inv_freq, DEV)
    step.page_table.copy_(page_tables(rng, S, 12, 13))
    on = lambda x: torch.tensor(np.asarray(x), dtype=torch.float32, device=DEV)
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

    # the prompts, but for their last token, which is the first step's root (a prompt of one token leaves nothing)
    start = np.concatenate([[0], np.cumsum([len(p) - 1 for p in prompts])])
    step.begin(torch.tensor(start, dtype=torch.int32, device=DEV))
    forward([t for p in prompts for t in p[:-1]])
    step.commit()
    assert step.kv_len.tolist() == [len(p) - 1 for p in prompts]
    done, accepted = [[] for _ in prompts], 0
    for _ in range(STEPS):
        nodes = rng.integers(0, g + 1, S).astype(np.int32)
        trees = [dc.random_tree(rng, g, D) for _ in range(S)]
        token, chunk = np.zeros((S, g), np.int32), []
        for s in range(S):
            parent, depth, _ = trees[s]
            right = {-1: True}
            taken = set()
            for n in range(g):
                a, at = int(parent[n]), len(done[s]) + int(depth[n]) - 1
                right[n] = right[a] and a not in taken and at < len(truth[s][0]) and bool(rng.random() < 0.6)
                if right[n]:
                    taken.add(a)
                    token[s, n] = truth[s][0][at]
                else:
                    token[s, n] = rng.integers(0, m.V)
            root = done[s][-1] if done[s] else prompts[s][-1]
            chunk.append([root] + token[s, :nodes[s]].tolist())
        tree = dict(node_token=torch.from_numpy(token), node_parent=torch.from_numpy(np.stack([t[0] for t in trees])),
                    node_depth=torch.from_numpy(np.stack([t[1] for t in trees])),
                    node_mask=torch.from_numpy(dc.words(np.stack([t[2] for t in trees]))), n_nodes=torch.from_numpy(nodes))
        tree = {n: x.to(DEV) for n, x in tree.items()}
        start = np.concatenate([[0], np.cumsum([len(c) for c in chunk])])
        step.begin(torch.tensor(start, dtype=torch.int32, device=DEV), tree)
        logits = forward(sum(chunk, []))
        target = torch.zeros((S, 1 + g, m.V), device=DEV)
        for s in range(S):
            target[s, :len(chunk[s])] = logits[start[s]:start[s + 1]]
        verdict = step.verify(tree, target, None, torch.zeros(S, device=DEV), torch.zeros((S, g), device=DEV), torch.zeros(S, device=DEV))
        step.commit()
        assert step.status() == 0
        n, got = verdict["accept_len"].tolist(), verdict["token"].tolist()
        for s in range(S):
            new = got[s][:n[s] + 1]
            assert got[s][n[s] + 1:] == [-1] * (D - n[s])
            assert new == truth[s][0][len(done[s]):len(done[s]) + len(new)]
            done[s] += new
            accepted += n[s]
    assert accepted > 0
    assert step.kv_len.tolist() == [len(p) - 1 + len(d) for p, d in zip(prompts, done)]
    step.close()


# ------------------------------------------------------------------ with the training pass's trees, against the oracle

def host_batch(step, trees=None, g=0):
    h = {n: x.cpu().numpy() for n, x in step.batch.items()}
    if trees is not None:
        words = h["node_mask"].view(np.uint64)
        h["node_mask"] = (words[..., np.arange(g) // 64] >> (np.arange(g) % 64).astype(np.uint64) & np.uint64(1)).astype(bool)
    return h


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,shape,page", [("bf16", (8, 2, 128), 24), ("f16", (6, 3, 64), 16), ("f32", (4, 2, 96), 5),
                                              ("bf16", (4, 4, 80), 7)])
def test_steps_with_the_trees_that_training_builds(dtype, shape, page):
    """gto_build_tree -> append and attention in two layers -> verification in the reward pass's row layout -> commit,
    three times, every call's outputs against the oracle's on the same inputs."""
    import harness
    from paper_2509_22134_b200 import binding as gto
    from paper_2509_22134_b200.runner import DecodeStep, draft_trees
    hq, hkv, dh = shape
    w = synth.Workload("step", B=8, V_draft=512, V_target=2048, D=4, k=4, g=20, dtype="f32", seed=21, sigma_t=1.0)
    p, data = harness.run_pass(w, DEV)
    rng = np.random.default_rng(7)
    S, g, layers, scale = w.B, w.g, 2, dh ** -0.5
    rope = 48 if dh == 96 else 64
    cfg = gto.make_decode_config(S=S, T=S * (g + 9), n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, page_size=page,
                                 n_pages=S * 30, max_pages=30, dtype=dtype, g=g, D=w.D, k=w.k, rope_dims=rope,
                                 softmax_scale=scale, V_draft=w.V_draft, V_target=w.V_target, logit_dtype="f32",
                                 flags=gto.GTO_DECODE_CONTEXT_ROWS)
    f = 10000.0 ** (-np.arange(rope // 2) / (rope // 2))
    step = DecodeStep(cfg, layers, f, DEV)
    step.page_table.copy_(page_tables(rng, S, 30, 30))
    on = lambda x: torch.tensor(x, device=DEV).to(step.k_cache.dtype)
    for turn in range(3):
        trees = draft_trees(p.tree, 0, S, turn % 2)
        lead = rng.integers(0 if turn else 1, 9, S)
        start = np.concatenate([[0], np.cumsum(lead + g)]).astype(np.int32)
        before = step.kv_len.cpu().numpy()
        step.begin(torch.from_numpy(start).to(DEV), trees)
        batch = host_batch(step, trees, g)
        n, T = int(start[-1]), int(start[-1]) + 2
        used = np.zeros((cfg.n_pages, page), bool)
        for s in range(S):
            pages, place = dec.slots(batch, s, np.arange(batch["kv_len"][s]), page)
            used[pages, place] = True
        for i in range(layers):
            x = dc.round_to(rng.normal(size=(T, hq + 2 * hkv, dh)), dtype)
            k0, v0 = step.k_cache[i].double().cpu().numpy(), step.v_cache[i].double().cpu().numpy()
            want_q, want_k, want_v = dec.append(batch, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], k0, v0, page, f, g)
            y = on(x)
            out = torch.full((T, hq, dh), 5.0, dtype=y.dtype, device=DEV)
            lse = torch.full((T, hq), 5.0, device=DEV)
            step.attend(i, y[:, :hq], y[:, hq:hq + hkv], y[:, hq + hkv:], out, lse)
            k1, v1 = step.k_cache[i].double().cpu().numpy(), step.v_cache[i].double().cpu().numpy()
            assert np.array_equal(v1, want_v)
            assert np.all(np.abs(k1 - want_k) <= append_tolerance(dtype, want_k))
            q1 = step.q_rotated.double().cpu().numpy()[:T]
            q1[n:] = 0.0                    # rows of no sequence, never written
            assert np.all(np.abs(q1[:n] - want_q[:n]) <= append_tolerance(dtype, want_q[:n]))
            c = SimpleNamespace(host=batch, q=q1, k=k1, v=v1, page=page, g=g, used=used, dh=dh, dtype=dtype, n=n)
            compare_attention(c, scale, out, lse)
        target = data["target"][turn % 2].contiguous()
        temperature = np.where(np.arange(S) % 3 == 0, 0.0, 0.9).astype(np.float32)
        u_node, u_bonus = rng.random((S, g), dtype=np.float32), rng.random(S, dtype=np.float32)
        verdict = step.verify(trees, target, data["d2t"], *(torch.from_numpy(u).to(DEV) for u in (temperature, u_node, u_bonus)))
        d2t = None if data["d2t"] is None else data["d2t"].cpu().numpy()
        host = {name: trees[name].cpu().numpy() for name in ("node_parent", "node_token", "node_depth", "node_slot")}
        z = target.double().cpu().numpy()
        length, path = verdict["accept_len"].cpu().numpy(), verdict["path_node"].cpu().numpy()
        for s in range(S):
            rows = np.where((host["node_depth"][s] < w.D) & (host["node_slot"][s] >= 0),
                            1 + (host["node_depth"][s] - 1) * w.k + host["node_slot"][s], -1)
            want, ids, last, margin = dec.verify(host["node_parent"][s], host["node_token"][s], rows, z[s], float(temperature[s]),
                                                 u_node[s].astype(np.float64), float(u_bonus[s]), w.D, d2t)
            assert margin > 1e-9            # (the inputs are fixed: no decision of theirs is a tie)
            assert path[s, :length[s]].tolist() == want
            assert verdict["token"][s].tolist() == ids + [last] + [-1] * (w.D - len(ids))
        k0, v0 = step.k_cache.clone(), step.v_cache.clone()
        step.commit()
        for s in range(S):
            base = int(before[s] + lead[s])
            for j in range(length[s]):
                a, b = (tuple(int(y) for y in dec.slots(batch, s, base + e, page)) for e in (path[s, j], j))
                k0[:, b[0], b[1]] = k0[:, a[0], a[1]]
                v0[:, b[0], b[1]] = v0[:, a[0], a[1]]
        assert torch.equal(step.k_cache, k0) and torch.equal(step.v_cache, v0)
        assert step.kv_len.tolist() == (before + lead + length).tolist()
        assert step.status() == 0
    assert step.launches() > 0
    step.close()


# ------------------------------------------------------------------ graphs, streams, contexts, far addresses

SERVED = [("bf16", (8, 2, 128), 16), ("f32", (4, 2, 64), 16), ("f16", (4, 4, 64), 8)]


class Loop:
    """Decoding steps with buffers that stay, so that a step can be captured and replayed with other contents."""

    def __init__(self, dtype, shape, page, S=6, g=14, D=5, V=1024, stream=None):
        from paper_2509_22134_b200 import binding as gto
        from paper_2509_22134_b200.runner import DecodeStep
        self.gto, self.shape, self.S, self.g, self.D, self.V = gto, shape, S, g, D, V
        hq, hkv, dh = shape
        self.T = S * (g + 300)
        cfg = gto.make_decode_config(S=S, T=self.T, n_q_heads=hq, n_kv_heads=hkv, head_dim=dh, page_size=page, n_pages=S * 120,
                                     max_pages=120, dtype=dtype, g=g, D=D, V_draft=V, V_target=V, logit_dtype=dtype)
        self.step = DecodeStep(cfg, 2, 10000.0 ** (-np.arange(dh // 2) / (dh // 2)), DEV)
        self.step.page_table.copy_(page_tables(np.random.default_rng(1), S, 120, 120))
        t = self.step.k_cache.dtype
        zero = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device=DEV)
        self.buf = dict(q_start=zero(S + 1), n_nodes=zero(S), node_token=zero(S, g), node_parent=zero(S, g), node_depth=zero(S, g),
                        node_mask=zero(S, g, 1, dt=torch.int64), x=zero(self.T, hq + 2 * hkv, dh, dt=t),
                        target=zero(S, 1 + g, V, dt=t), temperature=zero(S, dt=torch.float32),
                        u_node=zero(S, g, dt=torch.float32), u_bonus=zero(S, dt=torch.float32))
        self.out = [zero(self.T, hq, dh, dt=t) for _ in range(2)]
        self.lse = zero(self.T, hq, dt=torch.float32)

    def fill(self, seed):
        """The inputs of one step: leads of 0 to 300 tokens, trees of 0 to g nodes."""
        rng = np.random.default_rng(seed)
        S, g, b = self.S, self.g, self.buf
        lead = rng.choice([0, 1, 1, 1, 2, 40, 300 if seed % 3 == 0 else 1], S)
        nodes = rng.integers(0, g + 1, S)
        trees = [dc.random_tree(rng, g, self.D) for _ in range(S)]
        new = dict(q_start=np.concatenate([[0], np.cumsum(lead + nodes)]), n_nodes=nodes,
                   node_token=rng.integers(0, self.V, (S, g)), node_parent=np.stack([t[0] for t in trees]),
                   node_depth=np.stack([t[1] for t in trees]), node_mask=dc.words(np.stack([t[2] for t in trees])),
                   x=rng.normal(size=tuple(b["x"].shape)), target=rng.normal(size=tuple(b["target"].shape)),
                   temperature=rng.choice([0.0, 1.0], S), u_node=rng.random((S, g)) * 2e-3, u_bonus=rng.random(S))
        for n, y in new.items():
            b[n].copy_(torch.from_numpy(np.ascontiguousarray(y)))

    def run(self):
        b, (hq, hkv, _) = self.buf, self.shape
        self.step.begin(b["q_start"], b)
        x = b["x"]
        for i in range(2):
            self.step.attend(i, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], self.out[i], self.lse)
        self.step.verify(b, b["target"], None, b["temperature"], b["u_node"], b["u_bonus"])
        self.step.commit()

    def state(self):
        s = self.step
        return [x.clone() for x in (*self.out, self.lse, s.kv_len, s.k_cache, s.v_cache, *s.verdict.values())]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b, strict=True))


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(len(SERVED)))
def test_a_captured_step_replays_with_other_lengths_and_trees(which):
    eager, captured = Loop(*SERVED[which]), Loop(*SERVED[which])
    want = []
    for seed in range(6):
        eager.fill(seed)
        eager.run()
        want.append(eager.state())
    assert eager.step.status() == 0
    captured.fill(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.run()
    for seed in range(6):
        captured.fill(seed)
        graph.replay()
        assert same(captured.state(), want[seed]), seed
    assert captured.step.status() == 0
    del graph


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(len(SERVED)))
def test_two_contexts_on_two_streams_at_once(which):
    """Each gives the bits that it gives alone; equal calls give equal bits."""
    alone = []
    for first in (10, 20):
        a = Loop(*SERVED[which])
        for seed in range(first, first + 3):
            a.fill(seed)
            a.run()
        alone.append(a.state())
    both = [Loop(*SERVED[which]) for _ in range(2)]
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(3):
        for a, first in zip(both, (10, 20)):
            a.fill(first + i)
        torch.cuda.synchronize()
        for a, s in zip(both, streams):
            with torch.cuda.stream(s):
                a.run()
        torch.cuda.synchronize()
    for a, want in zip(both, alone):
        assert a.step.status() == 0
        assert same(a.state(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_major", [False, True])
def test_pages_behind_four_gigabytes(dtype, head_major):
    """A pool of more than 2^31 elements, whose last pages are the ones in use: the bits of a small pool's calls."""
    from paper_2509_22134_b200 import binding as gto
    g, hkv, dh, page = 12, 8, 128, 64
    c = dc.Case([13, 30, 1], [13, 700, 90], 16, hkv, dh, page, dtype, g, 4, [12, 12, 0], seed=3, poison=1.0, head_major=head_major)
    far_pages = (1 << 31) // (page * hkv * dh) + c.n_pages + 5
    shape = (far_pages, hkv, page, dh) if head_major else (far_pages, page, hkv, dh)
    far = {}
    for n in ("k", "v"):
        pool = torch.empty(shape, dtype=dc.TORCH[dtype], device=DEV)
        far[n] = pool.permute(0, 2, 1, 3) if head_major else pool
        far[n][-c.n_pages:].copy_(c.dk if n == "k" else c.dv)
    batch = dict(c.batch)
    batch["page_table"] = torch.where(c.batch["page_table"] < c.n_pages, c.batch["page_table"] + (far_pages - c.n_pages),
                                      c.batch["page_table"])
    cfg = gto.make_decode_config(S=c.S, T=c.T, n_q_heads=16, n_kv_heads=hkv, head_dim=dh, page_size=page, n_pages=far_pages,
                                 max_pages=c.max_pages, dtype=dtype, g=g, D=4)
    f = torch.tensor(10000.0 ** (-np.arange(dh // 2) / (dh // 2)), device=DEV)
    qkv = c.tensor(c.rng.normal(size=(c.T, 16 + 2 * hkv, dh)))
    verdict = dict(accept_len=torch.tensor([2, 3, 0], dtype=torch.int32, device=DEV),
                   path_node=torch.tensor([[3, 7, -1, -1], [1, 2, 11, -1], [-1] * 4], dtype=torch.int32, device=DEV),
                   token=torch.zeros((3, 5), dtype=torch.int32, device=DEV))
    got = []
    for ctx, b, k, v in ((c.ctx(gto), c.batch, c.dk, c.dv), (gto.gto_decode_create(cfg, 0), batch, far["k"], far["v"])):
        q_out, out = torch.zeros((c.T, 16, dh), dtype=qkv.dtype, device=DEV), torch.zeros((c.T, 16, dh), dtype=qkv.dtype, device=DEV)
        new_len = torch.zeros(3, dtype=torch.int32, device=DEV)
        gto.gto_kv_append(ctx, b, qkv[:, :16], qkv[:, 16:16 + hkv], qkv[:, 16 + hkv:], q_out, k, v, f)
        gto.gto_tree_attention(ctx, b, q_out, k, v, out)
        gto.gto_kv_commit(ctx, b, verdict, k, v, new_len)
        assert gto.gto_decode_status(ctx) == 0
        got.append((q_out, out, new_len, k[-c.n_pages:].clone(), v[-c.n_pages:].clone()))
    assert same(*got)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_of_several_hundred_thousand_entries(dtype):
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case([1, 3], [300001, 77], 4, 1, 64, 128, dtype, seed=8, poison=None)
    ctx = c.ctx(gto, softmax_scale=0.125)
    out = torch.full((c.T, c.hq, c.dh), 5.0, dtype=c.dq.dtype, device=DEV)
    z = torch.full((c.T, c.hq), 5.0, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
    assert gto.gto_decode_status(ctx) == 0
    compare_attention(c, 0.125, out, z, c.attention_on_device(0.125))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_on_another_stream_than_the_current_one(dtype):
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case([20, 1], [50, 400], 8, 2, 64, 16, dtype, seed=4)
    ctx = c.ctx(gto, softmax_scale=0.125)
    out = torch.full((c.T, c.hq, c.dh), 5.0, dtype=c.dq.dtype, device=DEV)
    z = torch.full((c.T, c.hq), 5.0, device=DEV)
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z, stream=side)
    assert gto.gto_decode_status(ctx, side) == 0
    compare_attention(c, 0.125, out, z)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_calls_without_sequences_or_tokens_do_nothing(dtype):
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case([0, 0], [5, 0], 4, 2, 64, 16, dtype, 4, 2, seed=4, spare=2)
    ctx = c.ctx(gto)
    out = torch.full((c.T, 4, 64), 5.0, dtype=c.dq.dtype, device=DEV)
    k, v = c.dk.clone(), c.dv.clone()
    f = torch.tensor(10000.0 ** (-np.arange(32) / 32), device=DEV)
    gto.gto_kv_append(ctx, c.batch, c.dq, c.dq[:, :2], c.dq[:, :2], out, k, v, f)
    gto.gto_tree_attention(ctx, c.batch, c.dq, k, v, out)
    none = {"q_start": c.batch["q_start"][:1], "kv_len": c.batch["kv_len"][:0], "page_table": c.batch["page_table"][:0]}
    empty = c.dq[:0]
    gto.gto_kv_append(ctx, none, empty, empty[:, :2], empty[:, :2], out[:0], k, v, f)
    gto.gto_tree_attention(ctx, none, empty, k, v, out[:0])
    assert gto.gto_decode_status(ctx) == 0
    assert torch.all(out == 5.0)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(k.view(bits), c.dk.view(bits)) and torch.equal(v.view(bits), c.dv.view(bits))


# ------------------------------------------------------------------ where the kernels choose other variants

@pytest.mark.gpu
@pytest.mark.parametrize("dtype,V", [("f32", 393216), ("bf16", 786432), ("f16", 700000)])
@pytest.mark.parametrize("S", [2, 41])
def test_verify_the_longest_rows(dtype, V, S):
    """Rows of up to 1.5 MB, few trees and many."""
    from paper_2509_22134_b200 import binding as gto
    from test_decode_gpu import check_verdict, run_verify, verify_case
    if S > 2:
        V = V // 128 * 8          # (16-byte rows)
    c = verify_case(np.random.default_rng(V + S), S, 5, 3, V, V, dtype)
    ctx, out = run_verify(gto, c, 3, V, V, dtype)
    assert gto.gto_decode_status(ctx) == 0
    for s in range(S):
        check_verdict(c, s, out, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("q_lens,kv_lens,shape,page,g", [
    ([700], [900], (32, 8, 64), 16, 0), ([40, 61, 200, 61], [45, 300, 201, 77], (32, 16, 256), 5, 40),   # two CTAs a unit
    ([61, 61], [400, 90], (16, 2, 128), 9, 60), ([1], [1000], (2, 1, 256), 3, 0)])                        # four, eight
def test_fp32_attention_with_other_numbers_of_ctas(q_lens, kv_lens, shape, page, g):
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case(q_lens, kv_lens, *shape, page, "f32", g, 6, seed=len(q_lens))
    scale = c.dh ** -0.5
    ctx = c.ctx(gto, softmax_scale=scale)
    out = torch.full((c.T, c.hq, c.dh), 5.0, device=DEV)
    z = torch.full((c.T, c.hq), 5.0, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
    assert gto.gto_decode_status(ctx) == 0
    bare = SimpleNamespace(**{**vars(c), "k": np.where(c.used[..., None, None], c.k, 0.0), "v": np.where(c.used[..., None, None], c.v, 0.0)})
    compare_attention(c, scale, out, z, dc.Case.attention_on_device(bare, scale))


@pytest.mark.gpu
def test_append_refuses_rotated_queries_over_keys_or_values():
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case([3], [10], 2, 2, 64, 16, "bf16", seed=1, poison=0.0)
    ctx = c.ctx(gto)
    f = torch.ones(32, dtype=torch.float64, device=DEV)
    k, v = torch.zeros_like(c.dq), torch.zeros_like(c.dq)
    for over in (k, v):
        with pytest.raises(gto.GtoError) as e:
            gto.gto_kv_append(ctx, c.batch, c.dq, k, v, over, c.dk, c.dv, f)
        assert e.value.code == 1
    assert gto.gto_decode_launch_count(ctx) == 0


@pytest.mark.gpu
def test_a_page_shared_by_two_sequences_is_read_by_both():
    """A common prompt's pages in two rows of the table; each sequence's own entries behind it."""
    from paper_2509_22134_b200 import binding as gto
    for dtype in ("bf16", "f32"):
        c = dc.Case([2, 2], [70, 70], 8, 2, 64, 16, dtype, seed=6, poison=None)
        c.host["page_table"][1, :4] = c.host["page_table"][0, :4]
        c.batch["page_table"].copy_(torch.from_numpy(c.host["page_table"]))
        ctx = c.ctx(gto, softmax_scale=0.125)
        out = torch.full((c.T, c.hq, c.dh), 5.0, dtype=c.dq.dtype, device=DEV)
        z = torch.full((c.T, c.hq), 5.0, device=DEV)
        gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
        assert gto.gto_decode_status(ctx) == 0
        compare_attention(c, 0.125, out, z)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_sequences_than_a_cta_has_threads(dtype):
    """1000 sequences, some without tokens, some with trees: the cut of the work goes through several of a thread's."""
    from paper_2509_22134_b200 import binding as gto
    rng = np.random.default_rng(12)
    S, g = 1000, 5
    nodes = rng.integers(0, g + 1, S)
    lead = rng.choice([0, 1, 1, 1, 3], S)
    nodes[lead == 0] = 0
    q_lens = (lead + nodes).tolist()
    kv_lens = [q + int(rng.integers(0, 200)) for q in q_lens]
    c = dc.Case(q_lens, kv_lens, 4, 2, 64, 8, dtype, g, 3, nodes, seed=3, poison=None)
    ctx = c.ctx(gto, softmax_scale=0.125)
    out = torch.full((c.T, c.hq, c.dh), 5.0, dtype=c.dq.dtype, device=DEV)
    z = torch.full((c.T, c.hq), 5.0, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
    assert gto.gto_decode_status(ctx) == 0
    compare_attention(c, 0.125, out, z, c.attention_on_device(0.125))


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,dh", [(128, 1, 128), (100, 1, 64), (192, 2, 128), (256, 2, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_many_query_heads_on_a_key_head(dtype, hq, hkv, dh):
    """A token's heads fill a row tile, or pass its end."""
    from paper_2509_22134_b200 import binding as gto
    c = dc.Case([1, 4, 9, 0, 2], [700, 4, 90, 3, 65], hq, hkv, dh, 16, dtype, 8, 3, [0, 3, 8, 0, 1], seed=hq, poison=None)
    scale = dh ** -0.5
    ctx = c.ctx(gto, softmax_scale=scale)
    out = torch.full((c.T, hq, dh), 5.0, dtype=c.dq.dtype, device=DEV)
    z = torch.full((c.T, hq), 5.0, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=z)
    assert gto.gto_decode_status(ctx) == 0
    compare_attention(c, scale, out, z, c.attention_on_device(scale))
