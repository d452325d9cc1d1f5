"""The operators of one decoding step over a draft tree, as cases to measure and to compare.

A step puts the keys and values of a chunk of new tokens into a paged cache, attends over the cache and
the chunk, judges the drafted tokens by the target model's probabilities and keeps the cache entries of
the accepted ones.  A chunk is any number of ordinary tokens ("lead": the last sampled token, or a piece of
a prompt) followed by the nodes of a draft tree; a plain decoding step is a chunk of one token.

With `own` false `run` computes an operator in elementary torch operations, with `own` true it calls the
library.  Sizes are those of the models this repository has workloads for: 32 query / 8 key heads of 128
(LLaMA-3.1-8B, Qwen3-8B), 40 / 40 (Vicuna-13B), 64 / 8 (LLaMA-3.3-70B), trees of 60 nodes and depth 7,
vocabularies of 32 000, 128 256 and 151 936.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ cases
def listed():
    heads8b = dict(hq=32, hkv=8, dh=128)
    return [
        # one user, one token: what a plain decoding step costs when nothing else runs
        dict(name="append-one", op="append", S=1, lead=1, ragged=False, g=0, D=1, ctx=777, page=16, dtype="bf16",
             norm=False, inter=False, rope=128, theta=500000.0, **heads8b),
        # a batch of trees of a model with normalised queries and keys
        dict(name="append-trees", op="append", S=64, lead=1, ragged=False, g=60, D=7, ctx=2000, page=64, dtype="bf16",
             norm=True, inter=False, rope=128, theta=1000000.0, **heads8b),
        # prompts of several users, as many key as query heads, fp16
        dict(name="append-prompts", op="append", S=8, lead=4000, ragged=True, g=0, D=1, ctx=500, page=32, dtype="f16",
             norm=False, inter=False, rope=128, theta=10000.0, hq=40, hkv=40, dh=128),
        # one user, one token, an 8000-token context: latency, the cache has to be split to fill the device
        dict(name="attn-one", op="attn", S=1, lead=1, ragged=False, g=0, D=1, ctx=8000, page=16, dtype="bf16", **heads8b),
        # a full batch of single tokens: the cache is read once, nothing else counts
        dict(name="attn-batch", op="attn", S=128, lead=1, ragged=False, g=0, D=1, ctx=6000, page=64, dtype="bf16", **heads8b),
        # a batch of draft trees: 61 query rows x 4 heads on every cache entry
        dict(name="attn-trees", op="attn", S=32, lead=1, ragged=False, g=60, D=7, ctx=4000, page=64, dtype="bf16", **heads8b),
        # pieces of prompts over what is cached already: bound by the matrix products
        dict(name="attn-prompts", op="attn", S=4, lead=2048, ragged=True, g=0, D=1, ctx=6000, page=128, dtype="f16", **heads8b),
        # small full-precision model, small tree, narrow heads, short pages
        dict(name="attn-f32", op="attn", S=3, lead=2, ragged=False, g=12, D=3, ctx=300, page=16, dtype="f32",
             hq=8, hkv=2, dh=64),
        # one user's tree, one vocabulary
        dict(name="verify-one", op="verify", S=1, g=60, D=7, V=32000, Vd=32000, dtype="f16"),
        # a batch of trees, reduced draft vocabulary
        dict(name="verify-batch", op="verify", S=128, g=60, D=7, V=128256, Vd=32000, dtype="bf16"),
        # one user, all layers of the cache
        dict(name="commit-one", op="commit", S=1, g=60, D=7, ctx=1500, page=16, layers=32, dtype="bf16", hkv=8, dh=128),
        # a batch, all layers of the cache
        dict(name="commit-batch", op="commit", S=64, g=60, D=7, ctx=700, page=64, layers=32, dtype="bf16", hkv=8, dh=128),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    return dict(rng.choice([dict(hq=32, hkv=8, dh=128), dict(hq=64, hkv=8, dh=128), dict(hq=8, hkv=1, dh=128),
                            dict(hq=40, hkv=40, dh=128), dict(hq=16, hkv=4, dh=64), dict(hq=20, hkv=4, dh=128)]))


def _tree(rng):
    D = rng.choice([3, 4, 5, 6, 7, 8])
    return dict(D=D, g=rng.randint(D * D, 64 if D < 8 else 100))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "verify", "commit"])
    page = rng.choice([8, 16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "append":
        h, t = _heads(rng), dict(g=0, D=1)
        S = _log_int(rng, 1, 64)
        if rng.random() < 0.5:
            t, lead, ragged = _tree(rng), rng.randint(0, 3), False
        else:
            lead, ragged = _log_int(rng, 1, max(1, 20000 // S)), True
        return dict(op=op, S=S, lead=lead, ragged=ragged, ctx=_log_int(rng, 1, max(1, 100000 // S)), page=page,
                    dtype=rng.choice([dtype, "f32"]), norm=rng.random() < 0.5, inter=rng.random() < 0.3,
                    rope=rng.choice([h["dh"], h["dh"] // 2]), theta=rng.choice([10000.0, 500000.0, 1000000.0]), **t, **h)
    if op == "attn":
        h, kind = _heads(rng), rng.choice(["one", "tree", "chunk", "f32"])
        if kind == "f32":
            return dict(op=op, S=_log_int(rng, 1, 8), lead=rng.randint(1, 4), ragged=False, ctx=_log_int(rng, 1, 1000), page=page,
                        dtype="f32", **_tree(rng), **rng.choice([dict(hq=8, hkv=2, dh=64), dict(hq=6, hkv=6, dh=64), dict(hq=8, hkv=1, dh=128)]))
        if kind == "one":
            S = _log_int(rng, 1, 128)
            return dict(op=op, S=S, lead=1, ragged=False, g=0, D=1, ctx=_log_int(rng, 1, min(60000, 700000 * 8 // (S * h["hkv"]))),
                        page=page, dtype=dtype, **h)
        if kind == "tree":
            S = _log_int(rng, 1, 32)
            return dict(op=op, S=S, lead=rng.randint(0, 3), ragged=False, ctx=_log_int(rng, 1, min(30000, 120000 // S)),
                        page=page, dtype=dtype, **_tree(rng), **h)
        S = _log_int(rng, 1, 4)
        return dict(op=op, S=S, lead=_log_int(rng, 2, 2000), ragged=True, g=0, D=1, ctx=_log_int(rng, 1, 4000), page=page,
                    dtype=dtype, **h)
    if op == "verify":
        Vd, V = rng.choice([(32000, 32000), (32000, 128256), (151936, 151936)])
        t = _tree(rng)
        return dict(op=op, S=_log_int(rng, 1, 100 if V == 128256 else 50), V=V, Vd=Vd, dtype=rng.choice([dtype, "f32"]), **t)
    return dict(op=op, S=_log_int(rng, 1, 64), ctx=_log_int(rng, 1, 700), page=page, layers=_log_int(rng, 1, 32), dtype=dtype,
                **_tree(rng), **rng.choice([dict(hkv=8, dh=128), dict(hkv=4, dh=64), dict(hkv=1, dh=128)]))


# ------------------------------------------------------------------ what a case's batch looks like
def _spread(s, S):
    """In (0, 1], 1 for the first sequence: a batch's lengths, the same for every seed."""
    return 1.0 - (s * 0.6180339887498949) % 1.0


def _lens(case):
    """(tokens of each chunk, entries of each sequence in the cache, the chunk's among them)."""
    S, g = case["S"], case["g"]
    lead = case.get("lead", 1)
    q = [(max(1, int(lead * _spread(s, S))) if case.get("ragged") else lead) + g for s in range(S)]
    return q, [q[s] + int(case["ctx"] * (0.25 + 0.75 * _spread(s + 1 if S > 1 else 0, S))) for s in range(S)]


def _widths(g, D):
    return [g // D + (1 if d < g % D else 0) for d in range(D)]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 2654435761 % (1 << 62) + 17)


def _normal(shape, gen, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(scale))
    return x


def _trees(case, gen):
    """Random trees, level by level: every node's parent is some node of the level above."""
    S, g, D = case["S"], case["g"], case["D"]
    parent = torch.full((S, g), -1, dtype=torch.int32, device=DEV)
    depth = torch.empty((S, g), dtype=torch.int32, device=DEV)
    first, prev = 0, None
    for d, w in enumerate(_widths(g, D)):
        if prev is not None:
            up = torch.randint(prev[0], prev[1], (S, w), generator=gen, device=DEV)
            parent[:, first:first + w] = torch.sort(up, 1).values.to(torch.int32)  # siblings stand together
        depth[:, first:first + w] = d + 1
        first, prev = first + w, (first, first + w)
    return parent, depth


def _ancestors(parent, D):
    """[S, g, g]: whether node a is node n or one of its ancestors."""
    S, g = parent.shape
    anc = torch.eye(g, dtype=torch.bool, device=DEV).repeat(S, 1, 1)
    at = parent.long()
    for _ in range(D):
        ok = at >= 0
        anc |= torch.nn.functional.one_hot(at.clamp(min=0), g).bool() & ok[:, :, None]
        at = torch.where(ok, torch.gather(parent.long(), 1, at.clamp(min=0)), at)
    return anc


def _words(anc):
    """Ancestor bits as 64-bit words, the form of the library's trees."""
    S, g, _ = anc.shape
    W = (g + 63) // 64
    full = torch.zeros((S, g, W * 64), dtype=torch.int64, device=DEV)
    full[:, :, :g] = anc.long()
    bit = torch.ones(64, dtype=torch.int64, device=DEV) << torch.arange(64, device=DEV)
    return (full.view(S, g, W, 64) * bit).sum(3)


def _batch(case, gen):
    q, kv = _lens(case)
    S, page = case["S"], case["page"]
    need = [-(-n // page) for n in kv]
    most = max(need)
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((S, most), dtype=torch.int32, device=DEV)
    first = 0
    for s in range(S):
        table[s, :need[s]] = order[first:first + need[s]]
        first += need[s]
    start = [0]
    for n in q:
        start.append(start[-1] + n)
    b = dict(q_start=torch.tensor(start, dtype=torch.int32, device=DEV), kv_len=torch.tensor(kv, dtype=torch.int32, device=DEV),
             page_table=table)
    anc = None
    if case["g"]:
        parent, b["node_depth"] = _trees(case, gen)
        anc = _ancestors(parent, case["D"])
        b["node_mask"] = _words(anc)
    return b, anc, dict(n=start[-1], T=start[-1] + 2, most_q=max(q), most_kv=max(kv), n_pages=n_pages, max_pages=most)


def _config(gto, case, size, **kw):
    return gto.make_decode_config(S=case["S"], T=size["T"], n_q_heads=case.get("hq", case["hkv"]), n_kv_heads=case["hkv"],
                                  head_dim=case["dh"], page_size=case["page"], n_pages=size["n_pages"],
                                  max_pages=size["max_pages"], dtype=case["dtype"], g=case["g"], D=case["D"], **kw)


# ------------------------------------------------------------------ inputs
def _inputs(case, seed):
    gen = _gen(seed)
    dt = _DT[case["dtype"]]
    s = dict(case=case)
    if case["op"] == "verify":
        S, g, D, V, Vd = (case[k] for k in ("S", "g", "D", "V", "Vd"))
        parent, depth = _trees(case, gen)
        # ids of the reduced vocabulary, increasing
        d2t = None if V == Vd else torch.sort(torch.randperm(V, generator=gen, device=DEV)[:Vd]).values.to(torch.int32)
        # distinct tokens for the nodes of a tree
        token = (torch.randint(0, Vd, (S, 1), generator=gen, device=DEV) + torch.arange(g, device=DEV) * (Vd // g)) % Vd
        token = token.to(torch.int32)
        z = _normal((S, 1 + g, V), gen, dt, 2.0)
        # what a drafter that agrees with the target most of the time proposes: the children of a context hold most
        # of its mass, the first the most
        ids = token.long() if d2t is None else d2t.long()[token.long()]
        older = (parent[:, None, :] == parent[:, :, None]) & torch.ones(g, g, dtype=torch.bool, device=DEV).tril(-1)
        rank = older.sum(2).float()
        lift = math.log(V) + 2.0 + 1.0 - 1.2 * rank + 0.5 * torch.randn((S, g), generator=gen, device=DEV)
        z.view(-1)[(torch.arange(S, device=DEV)[:, None] * (1 + g) + 1 + parent.long()) * V + ids] = lift.to(dt)
        temperature = 0.7 + 0.5 * torch.rand(S, generator=gen, device=DEV)
        temperature[3::4] = 0.0  # every fourth user decodes greedily
        s.update(tree=dict(node_token=token, node_parent=parent), target=z, d2t=d2t, temperature=temperature,
                 u_node=torch.rand((S, g), generator=gen, device=DEV), u_bonus=torch.rand(S, generator=gen, device=DEV),
                 anc=_ancestors(parent, D), depth=depth)
        return s
    b, anc, size = _batch(case, gen)
    s.update(batch=b, anc=anc, size=size)
    hkv, dh, page = case["hkv"], case["dh"], case["page"]
    pool = (size["n_pages"], page, hkv, dh)
    if case["op"] == "commit":
        s["k_cache"] = _normal((case["layers"],) + pool, gen, dt)
        s["v_cache"] = _normal((case["layers"],) + pool, gen, dt)
        S, g, D = case["S"], case["g"], case["D"]
        # a random path down some tree: at each level any node, the first level's away from where entries go
        w = _widths(g, D)
        first, path = 0, []
        for d in range(D):
            at = torch.randint(first, first + w[d], (S,), generator=gen, device=DEV)
            if d == 0:
                at = torch.where(at < D, 0, at)
            path.append(at)
            first += w[d]
        length = torch.randint(0, D + 1, (S,), generator=gen, device=DEV)
        path = torch.stack(path, 1)
        path = torch.where(torch.arange(D, device=DEV)[None] < length[:, None], path, -1)
        s["verdict"] = dict(accept_len=length.to(torch.int32), path_node=path.to(torch.int32),
                            token=torch.zeros((S, D + 1), dtype=torch.int32, device=DEV))
        s["new_len"] = torch.zeros(S, dtype=torch.int32, device=DEV)
        return s
    T, hq = size["T"], case["hq"]
    s["k_cache"], s["v_cache"] = _normal(pool, gen, dt), _normal(pool, gen, dt)
    if case["op"] == "append":
        # queries, keys and values are slices of one projection
        s["qkv"] = _normal((T, hq + 2 * hkv, dh), gen, dt)
        half = case["rope"] // 2
        s["inv_freq"] = case["theta"] ** (-torch.arange(half, dtype=torch.float64, device=DEV) / half)
        s["q_norm"] = (1 + 0.2 * torch.randn(dh, generator=gen, device=DEV)).to(dt) if case["norm"] else None
        s["k_norm"] = (1 + 0.2 * torch.randn(dh, generator=gen, device=DEV)).to(dt) if case["norm"] else None
        s["q_out"] = torch.zeros((T, hq, dh), dtype=dt, device=DEV)
    else:
        s["q"] = _normal((T, hq, dh), gen, dt, 1.5)
        s["out"] = torch.zeros((T, hq, dh), dtype=dt, device=DEV)
        s["lse"] = torch.zeros((T, hq), dtype=torch.float32, device=DEV)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2509_22134_b200 import binding as gto
        if case["op"] == "verify":
            cfg = gto.make_decode_config(S=case["S"], g=case["g"], D=case["D"], V_draft=case["Vd"], V_target=case["V"],
                                         logit_dtype=case["dtype"])
            s["verdict"] = gto.alloc_verdict(cfg, DEV)
        elif case["op"] == "append":
            cfg = _config(gto, case, s["size"], rope_dims=case["rope"],
                          flags=gto.GTO_DECODE_ROPE_INTERLEAVED if case["inter"] else 0)
        else:
            cfg = _config(gto, case, s["size"])
        # the library's context, as a program keeps it for as long as it decodes (it frees itself)
        s["ctx"] = gto.gto_decode_create(cfg, torch.cuda.current_device())
    return s


# ------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2509_22134_b200 import binding as gto
    case, op, ctx = s["case"], s["case"]["op"], s["ctx"]
    if op == "append":
        hq, hkv, x = case["hq"], case["hkv"], s["qkv"]
        gto.gto_kv_append(ctx, s["batch"], x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], s["q_out"], s["k_cache"],
                          s["v_cache"], s["inv_freq"], q_norm=s["q_norm"], k_norm=s["k_norm"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    if op == "attn":
        gto.gto_tree_attention(ctx, s["batch"], s["q"], s["k_cache"], s["v_cache"], s["out"], lse=s["lse"])
        return dict(out=s["out"], lse=s["lse"])
    if op == "verify":
        gto.gto_verify_tree(ctx, s["tree"], s["target"], s["d2t"], s["temperature"], s["u_node"], s["u_bonus"],
                            s["verdict"])
        return s["verdict"]
    gto.gto_kv_commit(ctx, s["batch"], s["verdict"], s["k_cache"], s["v_cache"], s["new_len"])
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], new_len=s["new_len"])


# ------------------------------------------------------------------ the plain forms
def _tokens(s):
    """Of every token of the batch: its sequence, its place in the chunk, the chunk's first cache entry."""
    b, n = s["batch"], s["size"]["n"]
    t = torch.arange(n, device=DEV)
    seq = torch.searchsorted(b["q_start"].long(), t, right=True) - 1
    place = t - b["q_start"].long()[seq]
    base = (b["kv_len"] - (b["q_start"][1:] - b["q_start"][:-1])).long()
    return seq, place, base


def _slots(s, seq, entry):
    """Rows of the cache (pages laid end to end) of cache entries `entry` of sequences `seq`."""
    page = s["case"]["page"]
    return s["batch"]["page_table"].long()[seq, entry // page] * page + entry % page


def _rotate(x, pos, s, weight):
    case = s["case"]
    x, rope = x.float(), case["rope"]
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + 1e-6) * weight.float()
    angle = pos.double()[:, None] * s["inv_freq"][None]  # 64 bits: far positions
    c, sn = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y, rest = x[:, :, :rope], x[:, :, rope:]
    if case["inter"]:
        a, b = y[:, :, 0::2], y[:, :, 1::2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], 3).flatten(2)
    else:
        a, b = y[:, :, :rope // 2], y[:, :, rope // 2:]
        y = torch.cat([a * c - b * sn, b * c + a * sn], 2)
    return torch.cat([y, rest], 2)


def _plain_append(s):
    case, n = s["case"], s["size"]["n"]
    hq, hkv, g = case["hq"], case["hkv"], case["g"]
    seq, place, base = _tokens(s)
    pos = base[seq] + place
    slot = _slots(s, seq, pos)
    if g:
        node = place - case["lead"]
        pos = torch.where(node >= 0, base[seq] + case["lead"] - 1 + s["batch"]["node_depth"].long()[seq, node.clamp(min=0)], pos)
    x = s["qkv"][:n]
    s["q_out"][:n] = _rotate(x[:, :hq], pos, s, s["q_norm"]).to(x.dtype)
    s["k_cache"].view(-1, hkv, case["dh"])[slot] = _rotate(x[:, hq:hq + hkv], pos, s, s["k_norm"]).to(x.dtype)
    s["v_cache"].view(-1, hkv, case["dh"])[slot] = x[:, hq + hkv:]
    return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_attn(s):
    case, size = s["case"], s["size"]
    S, hq, hkv, dh, lead, g = (case[k] for k in ("S", "hq", "hkv", "dh", "lead", "g"))
    n, nq, nkv = size["n"], size["most_q"], size["most_kv"]
    seq, place, base = _tokens(s)
    b, rep = s["batch"], hq // hkv
    entry = torch.arange(nkv, device=DEV)
    slot = _slots(s, torch.arange(S, device=DEV)[:, None], entry[None].expand(S, nkv))
    k = s["k_cache"].view(-1, hkv, dh)[slot].float().permute(0, 2, 3, 1)     # [S, hkv, dh, nkv]
    v = s["v_cache"].view(-1, hkv, dh)[slot].float().permute(0, 2, 1, 3)     # [S, hkv, nkv, dh]
    q = torch.zeros((S, nq, hq, dh), device=DEV)
    q[seq, place] = s["q"][:n].float()
    q = q.view(S, nq, hkv, rep, dh).permute(0, 2, 3, 1, 4).reshape(S, hkv, rep * nq, dh)
    i = torch.arange(nq, device=DEV)
    last = b["kv_len"].long()[:, None, None]
    see = (entry[None, None] <= base[:, None, None] + i[None, :, None]) & (entry[None, None] < last)   # [S, nq, nkv]
    if g:
        node = entry[None, :] - (base[:, None] + lead)                                                # [S, nkv]
        inside = torch.gather(s["anc"], 2, node.clamp(0, g - 1)[:, None, :].expand(S, g, nkv))
        tree = (node < 0)[:, None] | (inside & (node >= 0)[:, None] & (node < g)[:, None])
        see = torch.cat([see[:, :lead], tree], 1)
    x = (q @ k).mul_(1.0 / math.sqrt(dh)).view(S, hkv, rep, nq, nkv)
    x.masked_fill_(~see[:, None, None], -math.inf)
    top = x.amax(4, keepdim=True)
    top = torch.where(torch.isinf(top), 0.0, top)
    x = x.sub_(top).exp_()
    total = x.sum(4, keepdim=True)
    o = (x.view(S, hkv, rep * nq, nkv) @ v).view(S, hkv, rep, nq, dh) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0]
    s["out"][:n] = o.permute(0, 3, 1, 2, 4).reshape(S, nq, hq, dh)[seq, place].to(s["out"].dtype)
    s["lse"][:n] = lse.permute(0, 3, 1, 2).reshape(S, nq, hq)[seq, place]
    return dict(out=s["out"], lse=s["lse"])


def _plain_verify(s):
    """Every node of every tree judged at once, in 64 bits (a decision near a border must not fall to rounding)."""
    case = s["case"]
    S, g, D, V = (case[k] for k in ("S", "g", "D", "V"))
    parent, depth = s["tree"]["node_parent"].long(), s["depth"].long()
    token = s["tree"]["node_token"].long()
    ids = token if s["d2t"] is None else s["d2t"].long()[token]
    z, heat = s["target"], s["temperature"].double()
    cold = heat == 0
    heat = torch.where(cold, 1.0, heat)
    top = z.amax(2, keepdim=True)
    best = z.argmax(2)                                                       # the first of equal ones
    weight = z.double().sub_(top.double()).div_(heat[:, None, None]).exp_()   # [S, 1 + g, V]
    mass = weight.sum(2)
    row = parent + 1
    own_mass = torch.gather(mass, 1, row)
    p = weight[torch.arange(S, device=DEV)[:, None], row, ids] / own_mass
    sibling = parent[:, :, None] == parent[:, None, :]
    older = sibling & torch.ones(g, g, dtype=torch.bool, device=DEV).tril(-1)
    p = torch.where((older & (ids[:, :, None] == ids[:, None, :])).any(2), 0.0, p)
    left = 1.0 - (older.double() @ p[:, :, None])[..., 0]
    ok = torch.where(cold[:, None], torch.gather(best, 1, row) == ids, s["u_node"].double() * left < p)
    taken = ok & ~(older & ok[:, None, :]).any(2)
    reached = (~s["anc"] | taken[:, None, :]).all(2)                          # a node and all above it taken
    length = torch.where(reached, depth, 0).amax(1)
    level = torch.arange(1, D + 1, device=DEV)
    here = reached[:, None] & (depth[:, None] == level[None, :, None])         # [S, D, g]
    node = torch.where(here.any(2), here.long().argmax(2), -1)
    got = torch.where(node >= 0, torch.gather(ids, 1, node.clamp(min=0)), -1)
    last = torch.where(length > 0, torch.gather(node, 1, (length - 1).clamp(min=0)[:, None])[:, 0], -1)
    rest = weight[torch.arange(S, device=DEV), last + 1]                      # [S, V]
    out = (parent == last[:, None])                                           # the children of the last node: all refused
    rest = rest.scatter_reduce(1, ids, torch.where(out, 0.0, math.inf).double(), "amin")
    sums = rest.cumsum(1)
    bonus = (sums <= s["u_bonus"].double()[:, None] * sums[:, -1:]).sum(1).clamp(max=V - 1)
    bonus = torch.where(cold, torch.gather(best, 1, last[:, None] + 1)[:, 0], bonus)
    tokens = torch.full((S, D + 1), -1, dtype=torch.int64, device=DEV)
    tokens[:, :D] = got
    tokens.scatter_(1, length[:, None], bonus[:, None])
    return dict(accept_len=length.to(torch.int32), path_node=node.to(torch.int32), token=tokens.to(torch.int32))


def _plain_commit(s):
    case, b, v = s["case"], s["batch"], s["verdict"]
    S, D, L = case["S"], case["D"], case["layers"]
    base = (b["kv_len"] - (b["q_start"][1:] - b["q_start"][:-1])).long() + 1
    j = torch.arange(D, device=DEV)[None].expand(S, D)
    seq = torch.arange(S, device=DEV)[:, None].expand(S, D)
    src = torch.where(j < v["accept_len"][:, None], v["path_node"].long(), j)  # the others stay where they are
    to, frm = _slots(s, seq, base[:, None] + j).reshape(-1), _slots(s, seq, base[:, None] + src).reshape(-1)
    k, w = s["k_cache"].view(L, -1, case["hkv"], case["dh"]), s["v_cache"].view(L, -1, case["hkv"], case["dh"])
    k[:, to] = k[:, frm]
    w[:, to] = w[:, frm]
    s["new_len"].copy_(base + v["accept_len"])
    return dict(k_cache=s["k_cache"], v_cache=s["v_cache"], new_len=s["new_len"])


_PLAIN = dict(append=_plain_append, attn=_plain_attn, verify=_plain_verify, commit=_plain_commit)


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ work
def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "verify":
        # about three tokens accepted: four rows looked at, of D + 1 at most
        rows = case["S"] * 4
        return dict(bytes=rows * case["V"] * e, flops=rows * case["V"] * 3)
    q, kv = _lens(case)
    n, entry = sum(q), case["hkv"] * case["dh"] * e
    if case["op"] == "append":
        size = n * (case["hq"] + 2 * case["hkv"]) * case["dh"]
        return dict(bytes=2 * size * e, flops=size * 6)
    if case["op"] == "commit":
        # half of the longest path on average, read and written, keys and values of every layer
        return dict(bytes=case["S"] * case["D"] / 2 * case["layers"] * entry * 4, flops=0)
    pairs = 0
    for a, b in zip(q, kv):
        lead = a - case["g"]
        pairs += a * (b - a) + lead * (lead + 1) // 2 + case["g"] * (lead + case["D"] // 2 + 1)
    return dict(bytes=sum(kv) * entry * 2 + n * case["hq"] * (2 * case["dh"] * e + 4), flops=4 * pairs * case["hq"] * case["dh"])


# ------------------------------------------------------------------ the definitions, in 64 bits
def exact(case, seed):
    if case["op"] in ("verify", "commit"):
        return None  # tokens, and copies
    s = _inputs(case, seed)
    b, g, dh, hkv, hq = s["batch"], case["g"], case["dh"], case["hkv"], case["hq"]
    start, table = b["q_start"].tolist(), b["page_table"].long()
    kv, page = b["kv_len"].tolist(), case["page"]
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    if case["op"] == "append":
        qo = s["q_out"].double()
        for i in range(case["S"]):
            lo, hi = start[i], start[i + 1]
            first = kv[i] - (hi - lo)
            e = torch.arange(first, kv[i], device=DEV)
            pos = e.double()
            if g:
                pos[hi - lo - g:] = (first + hi - lo - g - 1) + b["node_depth"][i].double()
            turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), torch.outer(pos, s["inv_freq"]))[:, None]
            x = s["qkv"][lo:hi].double()

            def turned(h, w):
                if w is not None:
                    h = h / torch.sqrt(h.square().sum(2, keepdim=True) / dh + 1e-6) * w.double()
                r = h[..., :case["rope"]]
                if case["inter"]:
                    z = torch.view_as_complex(r.reshape(*r.shape[:2], -1, 2).contiguous()) * turn
                    r = torch.view_as_real(z).flatten(2)
                else:
                    z = torch.complex(*r.chunk(2, 2)) * turn
                    r = torch.cat([z.real, z.imag], 2)
                return torch.cat([r, h[..., case["rope"]:]], 2)

            qo[lo:hi] = turned(x[:, :hq], s["q_norm"])
            kc[table[i][e // page], e % page] = turned(x[:, hq:hq + hkv], s["k_norm"])
            vc[table[i][e // page], e % page] = x[:, hq + hkv:]
        return dict(q=qo, k_cache=kc, v_cache=vc)
    out, lse = s["out"].double(), s["lse"].double()
    for i in range(case["S"]):
        lo, hi = start[i], start[i + 1]
        m = hi - lo
        e = torch.arange(kv[i], device=DEV)
        k, v = kc[table[i][e // page], e % page], vc[table[i][e // page], e % page]
        hide = torch.ones(m, kv[i], dtype=torch.bool, device=DEV).triu(kv[i] - m + 1)
        if g:
            hide[m - g:, kv[i] - g:] = ~s["anc"][i]
        for h in range(hq):
            x = s["q"][lo:hi, h].double() @ k[:, h // (hq // hkv)].T / math.sqrt(dh)
            x = x.masked_fill(hide, -math.inf)
            z = torch.logsumexp(x, 1)
            lse[lo:hi, h] = z
            w = torch.exp(x - torch.where(torch.isinf(z), 0.0, z)[:, None])
            out[lo:hi, h] = w @ v[:, h // (hq // hkv)]
    return dict(out=out, lse=lse)
