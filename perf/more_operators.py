"""More operators of the decoding step, as cases to measure and to compare: tokens drawn under limits
(temperature, top-k, top-p, min-p), drafted trees verified under the same limits, and the pages of the cache
(forked, grown and given back, moved together).

With `own` false `run` computes an operator in elementary torch operations, with `own` true it calls the
library.  Sizes are those of the models this repository has workloads for: vocabularies of 32 000, 128 256 and
151 936, 8 key heads of 128 and 32 layers (LLaMA-3.1-8B, Qwen3-8B), trees of 60 nodes and depth 7.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_TINY = -1000.0 * math.log(2.0)  # weights below 2^-1000 of the largest are nothing


# ------------------------------------------------------------------ cases
def listed():
    cache = dict(layers=32, hkv=8, dh=128)
    return [
        # one user, the token after the prompt: latency
        dict(name="sample-one", op="sample", N=1, V=128256, dtype="bf16", kind="top_p", flat=1.3),
        # a full batch of users, each with settings of their own (greedy ones among them)
        dict(name="sample-batch", op="sample", N=512, V=128256, dtype="bf16", kind="mixed", flat=1.2),
        # roll-outs for training: the temperature alone, 8 draws from every prompt's row
        dict(name="sample-rollouts", op="sample", N=1024, V=32000, dtype="f16", kind="plain", flat=1.2, draws=8),
        # creative settings on full-precision logits: the limits leave thousands of tokens
        dict(name="sample-wide", op="sample", N=48, V=151936, dtype="f32", kind="wide", flat=1.05),
        # one user's tree
        dict(name="verify-limited-one", op="verify", S=1, g=60, D=7, V=32000, Vd=32000, dtype="f16", kind="top_p"),
        # a batch of trees, reduced draft vocabulary
        dict(name="verify-limited-batch", op="verify", S=64, g=60, D=7, V=128256, Vd=32000, dtype="bf16", kind="mixed"),
        # one prompt, four continuations
        dict(name="fork-one", op="fork", S=4, n=4, ctx=600, page=16),
        # 32 long prompts, 16 continuations each
        dict(name="fork-batch", op="fork", S=512, n=16, ctx=12000, page=16),
        # between two steps of a batch: what the trees did not need goes back, the next trees get room
        dict(name="resize-step", op="resize", S=256, n=1, ctx=3000, page=16, chunk=61, layers=1, hkv=8, dh=128, dtype="bf16"),
        # 16 prompts forked 4 times: the last page of each is copied before the continuations write into it
        dict(name="resize-forked", op="resize", S=64, n=4, ctx=2000, page=64, chunk=61, dtype="bf16", **cache),
        # a small pool of a small model
        dict(name="compact-small", op="compact", S=6, ctx=300, page=16, full=0.5, layers=4, hkv=2, dh=64, dtype="f32"),
        # a pool that many sequences have left: what is used moves to its front
        dict(name="compact-pool", op="compact", S=48, ctx=900, page=32, full=0.6, dtype="bf16", **cache),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "verify", "fork", "resize", "compact"])
    page = rng.choice([8, 16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    cache = dict(layers=_log_int(rng, 1, 32), **rng.choice([dict(hkv=8, dh=128), dict(hkv=4, dh=64), dict(hkv=1, dh=128)]))
    if op == "sample":
        V = rng.choice([32000, 128256, 151936, 8 * rng.randint(64, 16000)])
        most = (512 * 128256 * 2) // (V * (4 if dtype == "f32" else 2))
        return dict(op=op, N=_log_int(rng, 1, min(1024, most)), V=V, dtype=dtype, flat=round(rng.uniform(1.05, 2.0), 2),
                    kind=rng.choice(["mixed", "mixed", "plain", "top_p", "wide"]), draws=rng.choice([1, 1, 1, 4]))
    if op == "verify":
        Vd, V = rng.choice([(32000, 32000), (32000, 128256), (151936, 151936)])
        D = rng.choice([3, 4, 5, 6, 7, 8])
        return dict(op=op, S=_log_int(rng, 1, 64 if V == 128256 else 40), D=D, g=rng.randint(D * D, 64 if D < 8 else 100),
                    V=V, Vd=Vd, dtype=dtype, kind=rng.choice(["mixed", "top_p", "wide", "plain"]))
    if op == "fork":
        n = rng.randint(1, 16)
        return dict(op=op, S=n * _log_int(rng, 1, 512 // n), n=n, ctx=_log_int(rng, 1, 12000), page=page)
    if op == "resize":
        n = rng.choice([1, 2, 3, 4, 8])
        return dict(op=op, S=n * _log_int(rng, 1, 64 // n), n=n, ctx=_log_int(rng, 1, 2000), page=min(page, 64),
                    chunk=rng.choice([1, 7, 61, 300]), dtype=dtype if dtype != "f32" else "bf16", **cache)
    return dict(op=op, S=_log_int(rng, 1, 48), ctx=_log_int(rng, 1, 1200), page=min(page, 64), full=round(rng.uniform(0.2, 0.95), 2),
                dtype=dtype if dtype != "f32" else "f16", **cache)


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 2654435761 % (1 << 62) + 29)


def _normal(shape, gen, dtype, scale=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 28):
        part = flat[i:i + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(scale))
    return x


def _uniform(n, gen, lo, hi):
    return lo + (hi - lo) * torch.rand(n, generator=gen, device=DEV)


def _limits(kind, n, gen):
    """Settings of n users."""
    if kind == "plain":
        return dict(temperature=_uniform(n, gen, 0.7, 1.2))
    if kind == "top_p":
        return dict(temperature=_uniform(n, gen, 0.6, 1.0), top_p=_uniform(n, gen, 0.85, 0.97))
    if kind == "wide":
        return dict(temperature=_uniform(n, gen, 1.0, 1.4), top_k=torch.randint(2000, 20000, (n,), generator=gen, device=DEV, dtype=torch.int32),
                    top_p=_uniform(n, gen, 0.95, 1.0), min_p=_uniform(n, gen, 0.0, 2e-4))
    temperature = _uniform(n, gen, 0.6, 1.1)
    top_k = torch.randint(1, 200, (n,), generator=gen, device=DEV, dtype=torch.int32)
    top_p, min_p = _uniform(n, gen, 0.8, 1.0), _uniform(n, gen, 0.01, 0.1)
    temperature[3::8] = 0.0  # every eighth decodes greedily
    top_k[0::2] = 0          # half of them go without top-k, half without top-p, three in four without min-p
    top_p[1::4] = 1.0
    top_p[2::4] = 1.0
    min_p[torch.arange(n, device=DEV) % 4 != 2] = 0.0
    return dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


def _logits(N, V, flat, gen, dt):
    """Rows whose probabilities fall with a power of their rank, as a language model's do; the power varies by row."""
    z = torch.empty((N, V), dtype=dt, device=DEV)
    power = _uniform(N, gen, flat, flat + 0.9)
    step = max(1, (1 << 27) // V)
    for i in range(0, N, step):
        part = z[i:i + step]
        rank = torch.rand(part.shape, generator=gen, device=DEV).mul_(V).add_(1.0)
        noise = torch.randn(part.shape, generator=gen, device=DEV)
        part.copy_(14.0 - power[i:i + step, None] * rank.log_() + 0.3 * noise)
    return z


def _trees(case, gen):
    """Random trees, level by level: every node's parent is some node of the level above."""
    S, g, D = case["S"], case["g"], case["D"]
    parent = torch.full((S, g), -1, dtype=torch.int32, device=DEV)
    first, prev = 0, None
    for w in [g // D + (1 if d < g % D else 0) for d in range(D)]:
        if prev is not None:
            up = torch.randint(prev[0], prev[1], (S, w), generator=gen, device=DEV)
            parent[:, first:first + w] = torch.sort(up, 1).values.to(torch.int32)
        first, prev = first + w, (first, first + w)
    return parent


def _spread(s, S):
    """In (0, 1], 1 for the first: a batch's lengths, the same for every seed."""
    return 1.0 - (s * 0.6180339887498949) % 1.0


def _prompt_lens(case):
    n = case.get("n", 1)
    return [max(1, int(case["ctx"] * (0.25 + 0.75 * _spread(s // n, case["S"] // n)))) for s in range(case["S"])]


def _inputs(case, seed):
    gen = _gen(seed)
    s = dict(case=case)
    if case["op"] == "sample":
        N, dt = case["N"], _DT[case["dtype"]]
        draws = case.get("draws", 1)
        R = -(-N // draws)
        s.update(logits=_logits(R, case["V"], case["flat"], gen, dt), limits=_limits(case["kind"], N, gen),
                 rows=(torch.arange(N, device=DEV) // draws).to(torch.int32) if draws > 1 else None,
                 u=torch.rand(N, generator=gen, device=DEV), token=torch.zeros(N, dtype=torch.int32, device=DEV),
                 logp=torch.zeros(N, device=DEV), n_kept=torch.zeros(N, dtype=torch.int32, device=DEV))
        return s
    if case["op"] == "verify":
        S, g, D, V, Vd = (case[k] for k in ("S", "g", "D", "V", "Vd"))
        parent = _trees(case, gen)
        d2t = None if V == Vd else torch.sort(torch.randperm(V, generator=gen, device=DEV)[:Vd]).values.to(torch.int32)
        token = (torch.randint(0, Vd, (S, 1), generator=gen, device=DEV) + torch.arange(g, device=DEV) * (Vd // g)) % Vd
        token = token.to(torch.int32)
        z = _normal((S, 1 + g, V), gen, _DT[case["dtype"]], 2.0)
        # a drafter that agrees with the target most of the time: the children of a context hold most of its mass
        ids = token.long() if d2t is None else d2t.long()[token.long()]
        older = (parent[:, None, :] == parent[:, :, None]) & torch.ones(g, g, dtype=torch.bool, device=DEV).tril(-1)
        lift = math.log(V) + 3.0 - 1.2 * older.sum(2).float() + 0.5 * torch.randn((S, g), generator=gen, device=DEV)
        z.view(-1)[(torch.arange(S, device=DEV)[:, None] * (1 + g) + 1 + parent.long()) * V + ids] = lift.to(z.dtype)
        s.update(tree=dict(node_token=token, node_parent=parent), target=z, d2t=d2t, limits=_limits(case["kind"], S, gen),
                 u_node=torch.rand((S, g), generator=gen, device=DEV), u_bonus=torch.rand(S, generator=gen, device=DEV))
        return s
    # a pool in the middle of its life: sequences over shuffled pages, and free pages between them
    S, page, n = case["S"], case["page"], case.get("n", 1)
    lens = _prompt_lens(case)
    chunk = case.get("chunk", 0)
    most = max(-(-(L + chunk) // page) for L in lens) + 1
    first = [s_ % n == 0 for s_ in range(S)]  # the prompts; the others continue them
    need = [-(-L // page) if f else 0 for L, f in zip(lens, first)]
    fresh = sum(-(-(L + chunk) // page) - L // page for L in lens)
    n_pages = int(sum(need) / case["full"]) + 1 if "full" in case else sum(need) + fresh + sum(need) // 4 + 8
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((S, most), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i in range(S):
        table[i, :need[i]] = order[at:at + need[i]]
        at += need[i]
    i32 = dict(dtype=torch.int32, device=DEV)
    s["size"] = dict(n_pages=n_pages, max_pages=most)
    s["pool"] = dict(page_table=table, kv_len=torch.tensor([L if f else 0 for L, f in zip(lens, first)], **i32),
                     held=torch.tensor(need, **i32),
                     ref_count=torch.bincount(order[:at].long(), minlength=n_pages).to(torch.int32))
    s["parent"] = torch.tensor([i - i % n for i in range(S)], **i32)
    if case["op"] == "fork":
        return s
    pool = (case["layers"], n_pages, page, case["hkv"], case["dh"])
    s["k_cache"], s["v_cache"] = _normal(pool, gen, _DT[case["dtype"]]), _normal(pool, gen, _DT[case["dtype"]])
    if case["op"] == "resize":
        s["keep"] = torch.tensor(lens, **i32)
        # (a prompt that others continue is not written any more)
        s["want"] = torch.tensor([-1 if n > 1 and f else L + chunk for L, f in zip(lens, first)], **i32)
    else:
        s.update(table_out=torch.zeros_like(table), ref_out=torch.zeros(n_pages, **i32), n_used=torch.zeros(1, **i32))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2509_22134_b200 import binding as gto
        if case["op"] == "sample":
            cfg = gto.make_decode_config(S=case["N"], V_draft=case["V"], V_target=case["V"], logit_dtype=case["dtype"])
        elif case["op"] == "verify":
            cfg = gto.make_decode_config(S=case["S"], g=case["g"], D=case["D"], V_draft=case["Vd"], V_target=case["V"],
                                         logit_dtype=case["dtype"])
            s["verdict"] = gto.alloc_verdict(cfg, DEV)
        else:
            hkv = case.get("hkv", 8)
            cfg = gto.make_decode_config(S=case["S"], T=case["S"], n_q_heads=hkv, n_kv_heads=hkv, head_dim=case.get("dh", 128),
                                         page_size=case["page"], dtype=case.get("dtype", "bf16"),
                                         flags=gto.GTO_DECODE_PAGES, **s["size"])
        # the library's context, as a program keeps it for as long as it decodes (it frees itself)
        s["ctx"] = gto.gto_decode_create(cfg, torch.cuda.current_device())
    return s


# ------------------------------------------------------------------ the library's calls
def _run_own(s):
    from paper_2509_22134_b200 import binding as gto
    op, ctx = s["case"]["op"], s["ctx"]
    if op == "sample":
        gto.gto_sample_tokens(ctx, s["logits"], s["limits"], s["u"], s["token"], logp=s["logp"], n_kept=s["n_kept"],
                              rows=s["rows"])
        return dict(token=s["token"], logp=s["logp"], n_kept=s["n_kept"])
    if op == "verify":
        gto.gto_verify_tree_limited(ctx, s["tree"], s["target"], s["d2t"], s["limits"], s["u_node"], s["u_bonus"], s["verdict"])
        return s["verdict"]
    pool = s["pool"]
    if op == "fork":
        gto.gto_pages_fork(ctx, pool, s["parent"])
        return pool
    if op == "resize":
        if s["case"]["n"] > 1:
            gto.gto_pages_fork(ctx, pool, s["parent"])
        else:
            gto.gto_pages_resize(ctx, pool, s["keep"], s["k_cache"], s["v_cache"])
        gto.gto_pages_resize(ctx, pool, s["want"], s["k_cache"], s["v_cache"])
        return dict(pool, k_cache=s["k_cache"], v_cache=s["v_cache"])
    gto.gto_pages_compact(ctx, pool, s["k_cache"], s["v_cache"], s["table_out"], s["ref_out"], s["n_used"])
    return dict(table=s["table_out"], ref=s["ref_out"], n_used=s["n_used"], k_cache=s["k_cache"], v_cache=s["v_cache"])


# ------------------------------------------------------------------ the plain forms
def _weights(z, limits):
    """Of rows z [n, V] and their settings: the weights (64 bits: sums of 10^5 terms next to a border) and which tokens are kept."""
    n, V = z.shape
    heat = limits["temperature"].double()
    heat = torch.where(heat == 0, 1.0, heat)
    x = (z.double() - z.amax(1, keepdim=True).double()) / heat[:, None]
    w = torch.where(x < _TINY, 0.0, x.exp())
    if len(limits) == 1:
        return w, z > -math.inf
    top, order = torch.sort(z, dim=1, descending=True, stable=True)  # equal ones: the lowest id first
    ws = torch.gather(w, 1, order)
    keep = top > -math.inf
    if "top_k" in limits:
        k = limits["top_k"].long()[:, None]
        keep &= (k <= 0) | (torch.arange(V, device=DEV)[None] < k)
    if "top_p" in limits:
        p = limits["top_p"].double()[:, None]
        sums = torch.where(keep, ws, 0.0).cumsum(1)
        before = torch.cat([torch.full((n, 1), -1.0, dtype=torch.float64, device=DEV), sums[:, :-1]], 1)
        keep &= (p >= 1) | (before < p * sums[:, -1:])
    if "min_p" in limits:
        keep &= ws >= limits["min_p"].double().clamp(0, 1)[:, None]
    return w, torch.zeros_like(keep).scatter_(1, order, keep)


def _draw(w, u):
    """Of weights [n, V]: the first id whose cumulative sum is above u times the whole."""
    sums = w.cumsum(1)
    return (sums <= u.double()[:, None] * sums[:, -1:]).sum(1).clamp(max=w.shape[1] - 1), sums[:, -1]


def _part(limits, i, j):
    return {k: v[i:j] for k, v in limits.items()}


def _plain_sample(s):
    N, V = s["case"]["N"], s["case"]["V"]
    step = max(1, (1 << 28) // V)
    for i in range(0, N, step):
        lim = _part(s["limits"], i, i + step)
        z = s["logits"][i:i + step] if s["rows"] is None else s["logits"][s["rows"][i:i + step].long()]
        w, keep = _weights(z, lim)
        w = torch.where(keep, w, 0.0)
        token, total = _draw(w, s["u"][i:i + step])
        logp = (torch.gather(w, 1, token[:, None])[:, 0] / total).log()
        cold = lim["temperature"] == 0
        s["token"][i:i + step] = torch.where(cold, z.argmax(1), token).to(torch.int32)
        s["logp"][i:i + step] = torch.where(cold, 0.0, logp).float()
        s["n_kept"][i:i + step] = torch.where(cold, 1, keep.sum(1)).to(torch.int32)
    return dict(token=s["token"], logp=s["logp"], n_kept=s["n_kept"])


def _plain_verify(s):
    """The walks of all sequences, level by level."""
    case = s["case"]
    S, g, D = case["S"], case["g"], case["D"]
    parent = s["tree"]["node_parent"].long()
    ids = s["tree"]["node_token"].long()
    ids = ids if s["d2t"] is None else s["d2t"].long()[ids]
    cold = s["limits"]["temperature"] == 0
    all_, at = torch.arange(S, device=DEV), torch.full((S,), -1, dtype=torch.int64, device=DEV)
    node, token = torch.full((S, D), -1, device=DEV), torch.full((S, D + 1), -1, device=DEV)
    length, going = torch.zeros(S, dtype=torch.int64, device=DEV), torch.ones(S, dtype=torch.bool, device=DEV)
    before = torch.ones(g, g, dtype=torch.bool, device=DEV).tril(-1)
    for _ in range(D + 1):
        z = s["target"][all_, at + 1]
        w, keep = _weights(z, s["limits"])
        w = torch.where(keep, w, 0.0)
        best = z.argmax(1)
        kid = parent == at[:, None]
        p = torch.where(kid, torch.gather(w, 1, ids) / w.sum(1, keepdim=True), 0.0)
        older = kid[:, None, :] & kid[:, :, None] & before
        p = torch.where((older & (ids[:, :, None] == ids[:, None, :])).any(2), 0.0, p)
        left = 1.0 - (older.double() @ p[:, :, None])[..., 0]
        ok = kid & torch.where(cold[:, None], ids == best[:, None], s["u_node"].double() * left < p)
        some, first = ok.any(1), ok.long().argmax(1)
        # where no child is accepted: the last token, from what is left
        rest = w.scatter_reduce(1, ids, torch.where(kid, 0.0, math.inf).double(), "amin")
        last = torch.where(cold, best, _draw(rest, s["u_bonus"])[0])
        here = torch.where(some, torch.gather(ids, 1, first[:, None])[:, 0], last)
        token[all_, length] = torch.where(going, here, token[all_, length])
        on = going & some
        slot = length.clamp(max=D - 1)
        node[all_, slot] = torch.where(on, first, node[all_, slot])
        at, length, going = torch.where(on, first, at), length + on, on
    return dict(accept_len=length.to(torch.int32), path_node=node.to(torch.int32), token=token.to(torch.int32))


def _count(pool, rows, upto, sign):
    """Adds `sign` to the counts of the pages in the first upto[s] slots of some rows."""
    used = torch.arange(rows.shape[1], device=DEV)[None] < upto[:, None]
    pool["ref_count"].index_add_(0, rows.clamp(min=0).long().flatten(), used.flatten().to(torch.int32), alpha=sign)


def _plain_fork(s):
    pool, page = s["pool"], s["case"]["page"]
    parent = s["parent"].long()
    move = parent != torch.arange(parent.numel(), device=DEV)
    src = parent.clamp(min=0)
    length = torch.where(parent >= 0, pool["kv_len"][src], 0)
    pages = (length + page - 1) // page
    slot = torch.arange(pool["page_table"].shape[1], device=DEV)[None]
    rows = torch.where(slot < pages[:, None], pool["page_table"][src], -1)
    _count(pool, pool["page_table"], torch.where(move, pool["held"], 0), -1)
    _count(pool, rows, torch.where(move, pages, 0), 1)
    pool["page_table"][:] = torch.where(move[:, None], rows, pool["page_table"])
    pool["kv_len"][:] = torch.where(move, length, pool["kv_len"])
    pool["held"][:] = torch.where(move, pages, pool["held"])
    return pool


def _plain_resize(s, want):
    case, pool = s["case"], s["pool"]
    page, table, ref = case["page"], pool["page_table"], pool["ref_count"]
    ask, held = want >= 0, pool["held"]
    need = torch.where(ask, (want + page - 1) // page, held)
    keep = torch.where(ask, torch.minimum(pool["kv_len"], want), pool["kv_len"])
    slot = torch.arange(table.shape[1], device=DEV)[None]
    inside = slot < torch.minimum(held, need)[:, None]
    shared = inside & (slot >= (keep // page)[:, None]) & (want > keep)[:, None] & (ref[table.clamp(min=0).long()] > 1)
    new = shared | ((slot >= held[:, None]) & (slot < need[:, None]))
    free = torch.nonzero(ref == 0)[:, 0]
    back = ask[:, None] & (slot < held[:, None]) & ((slot >= need[:, None]) | shared)
    was = table.clone()
    fresh = free[:int(new.sum())].to(torch.int32)  # in the order of sequences, then slots
    table[new] = fresh
    table[ask[:, None] & (slot >= need[:, None])] = -1
    gone = was[back].long()
    ref.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    ref[fresh.long()] = 1
    q, j = torch.nonzero(shared & (slot == (keep // page)[:, None]), as_tuple=True)
    q, j = q[(keep % page)[q] > 0], j[(keep % page)[q] > 0]
    inner = torch.arange(page, device=DEV)[None] < (keep % page)[q][:, None]  # the entries that go along
    frm, to = was[q, j].long(), table[q, j].long()
    for x in (s["k_cache"], s["v_cache"]):
        for layer in x:
            layer[to] = torch.where(inner[:, :, None, None], layer[frm], layer[to])
    pool["held"][:], pool["kv_len"][:] = need, keep


def _plain_resize_pass(s):
    if s["case"]["n"] > 1:
        _plain_fork(s)
    else:
        _plain_resize(s, s["keep"])
    _plain_resize(s, s["want"])
    return dict(s["pool"], k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_compact(s):
    pool, ref = s["pool"], s["pool"]["ref_count"]
    n = ref.numel()
    used = ref > 0
    n_used = used.sum()
    number = torch.arange(n, device=DEV)
    frm, to = torch.nonzero(used & (number >= n_used))[:, 0], torch.nonzero(~used & (number < n_used))[:, 0]
    where = number.clone()
    where[frm] = to
    table = pool["page_table"]
    s["table_out"][:] = torch.where(table >= 0, where[table.clamp(min=0).long()].to(torch.int32), table)
    s["ref_out"][:] = torch.where(used, ref, 0)
    s["ref_out"][to] = ref[frm]
    s["ref_out"][frm] = 0
    s["n_used"][0] = n_used
    for x in (s["k_cache"], s["v_cache"]):
        for layer in x:
            layer[to] = layer[frm]
    return dict(table=s["table_out"], ref=s["ref_out"], n_used=s["n_used"], k_cache=s["k_cache"], v_cache=s["v_cache"])


_PLAIN = dict(sample=_plain_sample, verify=_plain_verify, fork=_plain_fork, resize=_plain_resize_pass, compact=_plain_compact)


def run(state):
    if own:
        return _run_own(state)
    return _PLAIN[state["case"]["op"]](state)


# ------------------------------------------------------------------ work
def work(case):
    op = case["op"]
    if op == "sample":
        row = case["V"] * (4 if case["dtype"] == "f32" else 2)
        return dict(bytes=-(-case["N"] // case.get("draws", 1)) * row, flops=case["N"] * case["V"] * 3)
    if op == "verify":
        # about three tokens accepted: four rows looked at, of D + 1 at most
        rows = case["S"] * 4
        return dict(bytes=rows * case["V"] * (4 if case["dtype"] == "f32" else 2), flops=rows * case["V"] * 3)
    lens, page, n = _prompt_lens(case), case["page"], case.get("n", 1)
    if op == "fork":
        # table entries read and written, and their pages' counts
        return dict(bytes=sum(-(-L // page) for i, L in enumerate(lens) if i % n) * 16 + case["S"] * 16, flops=0)
    entry = case["layers"] * case["hkv"] * case["dh"] * (4 if case["dtype"] == "f32" else 2) * 2
    if op == "resize":
        kids = [L for i, L in enumerate(lens) if n == 1 or i % n]
        table = sum(-(-(L + case["chunk"]) // page) - L // page for L in kids) * 16 + case["S"] * 24
        if n > 1:
            table += sum(-(-L // page) for L in kids) * 16
        return dict(bytes=table + (2 * entry * sum(L % page for L in kids) if n > 1 else 0), flops=0)
    used = sum(-(-L // page) for L in lens)
    return dict(bytes=2 * entry * page * used * (1 - case["full"]) + used * 16, flops=0)


# ------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    if case["op"] != "sample":
        return None  # tokens, tables and copies
    s = _inputs(case, seed)
    lim = {k: v.double().tolist() for k, v in s["limits"].items()}
    u, logp = s["u"].double(), torch.zeros(case["N"], dtype=torch.float64, device=DEV)
    for i in range(case["N"]):
        heat = lim["temperature"][i]
        if heat == 0:
            continue
        z = s["logits"][i if s["rows"] is None else int(s["rows"][i])].double()
        lp = z / heat
        lp = lp - torch.logsumexp(lp, 0)
        # ids by falling probability; a prefix of them stays
        ids = torch.argsort(-z, stable=True)
        count = int((z > -math.inf).sum())
        if "top_k" in lim and lim["top_k"][i] > 0:
            count = min(count, int(lim["top_k"][i]))
        mass = lp[ids[:count]].exp()
        if "top_p" in lim and lim["top_p"][i] < 1:
            count = min(count, 1 + int((mass.cumsum(0) < lim["top_p"][i] * mass.sum()).sum()))
        if "min_p" in lim:
            count = max(1, min(count, int((mass / mass[0] >= lim["min_p"][i]).sum())))
        stay = torch.sort(ids[:count]).values
        p = torch.softmax(z[stay] / heat, 0)
        at = int(torch.searchsorted(p.cumsum(0), u[i:i + 1] * p.sum(), right=True).clamp(max=count - 1))
        logp[i] = torch.log_softmax(z[stay] / heat, 0)[at]
    return dict(token=None, logp=logp, n_kept=None)
