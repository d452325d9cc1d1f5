"""Batches whose tables contradict themselves: every call of a step skips the same sequences, and says so."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import decode_oracle as dec

DEV = "cuda:0"


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


FREQ = 10000.0 ** (-np.arange(32) / 32)


def attend(gto, ctx, c, fill=5.0):
    out = torch.full((c.T, c.hq, c.dh), fill, dtype=c.dq.dtype, device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out)
    return out.double().cpu().numpy()


def put(gto, ctx, c):
    x = c.tensor(c.rng.normal(size=(c.T, c.hq + 2 * c.hkv, c.dh)))
    q_out = torch.full((c.T, c.hq, c.dh), 7.0, dtype=x.dtype, device=DEV)
    k, v = c.dk.clone(), c.dv.clone()
    gto.gto_kv_append(ctx, c.batch, x[:, :c.hq], x[:, c.hq:c.hq + c.hkv], x[:, c.hq + c.hkv:], q_out, k, v,
                      torch.tensor(FREQ, device=DEV))
    return x, q_out, k, v


def set_starts(c, starts):
    c.batch["q_start"].copy_(torch.tensor(starts, dtype=torch.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("starts,good", [
    ([0, 5, 3, 3], (0,)),           # a chunk of -2 tokens
    ([0, 5, 900, 901], (0,)),       # chunks that begin or end behind the tokens
    ([0, 8, 4, 12], (0,)),          # two chunks with the same tokens, each possible by itself
    ([3, 0, 4, 12], ()),            # nothing is certain from the first sequence on
    ([0, 5, 5, -2147483648], (0, 1)),
])
def test_append_and_commit_report_sequences_that_contradict_themselves(gto, starts, good):
    c = dc.Case([5, 3, 4], [30, 40, 50], 4, 2, 64, 16, "bf16", seed=1, poison=0.0)
    set_starts(c, starts)
    lens = np.diff(np.array(starts, np.int64))
    c.host["q_start"] = np.concatenate([[0], np.cumsum([lens[s] if s in good else 0 for s in range(3)])]).astype(np.int32)
    ctx = c.ctx(gto)
    x, q_out, k, v = put(gto, ctx, c)
    assert gto.gto_decode_status(ctx) == 8
    y = x.double().cpu().numpy()
    want_q, want_k, want_v = dec.append(c.host, y[:, :4], y[:, 4:6], y[:, 6:], c.k, c.v, 16, FREQ)
    n = int(c.host["q_start"][-1])
    assert np.array_equal(v.double().cpu().numpy(), want_v)
    err = np.abs(k.double().cpu().numpy() - want_k)                   # (one rounding, as in test_append)
    assert np.all(err <= np.abs(want_k).max() * 2.0 ** -20 + dc.HALF_STEP["bf16"] * np.abs(want_k))
    err = np.abs(q_out.double().cpu().numpy()[:n] - want_q[:n])
    assert np.all(err <= np.abs(want_q[:n]).max(initial=0) * 2.0 ** -20 + dc.HALF_STEP["bf16"] * np.abs(want_q[:n]))
    assert torch.all(q_out[n:] == 7.0)
    verdict = dict(accept_len=torch.zeros(3, dtype=torch.int32, device=DEV), path_node=torch.zeros((3, 1), dtype=torch.int32, device=DEV),
                   token=torch.zeros((3, 2), dtype=torch.int32, device=DEV))
    new_len = torch.full((3,), -5, dtype=torch.int32, device=DEV)
    gto.gto_kv_commit(ctx, c.batch, verdict, k, v, new_len)
    assert gto.gto_decode_status(ctx) == 8
    assert new_len.tolist() == [[30, 40, 50][s] if s in good else -5 for s in range(3)]


@pytest.mark.gpu
def test_append_reports_a_sequence_without_tokens_whose_length_is_impossible(gto):
    c = dc.Case([3, 0], [30, 40], 4, 2, 64, 16, "bf16", seed=1, poison=0.0)
    ctx = c.ctx(gto)
    put(gto, ctx, c)
    assert gto.gto_decode_status(ctx) == 0
    for bad in (-1, c.max_pages * 16 + 1):
        c.batch["kv_len"][1] = bad
        put(gto, ctx, c)
        assert gto.gto_decode_status(ctx) == 8


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_skips_every_sequence_behind_a_decrease(gto, dtype):
    c = dc.Case([8, 3, 4], [30, 40, 50], 4, 2, 64, 16, dtype, seed=2, poison=0.0)
    ctx = c.ctx(gto)
    whole = attend(gto, ctx, c)
    assert gto.gto_decode_status(ctx) == 0
    set_starts(c, [0, 8, 4, 12])
    for _ in range(2):
        got = attend(gto, ctx, c)
        assert gto.gto_decode_status(ctx) == 8
        # (the cut of the work is another one: parts are joined elsewhere, so that bits may differ by a rounding)
        assert np.all(np.abs(got[:8] - whole[:8]) <= dc.HALF_STEP[dtype] * 4 * np.abs(whole[:8]).max())
        assert np.all(got[8:] == 5.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("at", [0, 1, 127, 128, 383, 384, 700, 999])
def test_a_decrease_among_a_thousand_sequences(gto, dtype, at):
    rng = np.random.default_rng(at)
    S = 1000
    q_lens = rng.integers(1, 4, S).tolist()
    c = dc.Case(q_lens, [q + int(rng.integers(0, 60)) for q in q_lens], 4, 2, 64, 8, dtype, seed=3, poison=0.0)
    ctx = c.ctx(gto)
    whole = attend(gto, ctx, c)
    start = c.host["q_start"].copy()
    start[at + 1:] -= start[at + 1] - start[at] + 1            # (sequence `at` has -1 tokens; what follows overlaps)
    set_starts(c, start)
    got = attend(gto, ctx, c)
    assert gto.gto_decode_status(ctx) == 8
    n = int(start[at])
    assert np.all(np.abs(got[:n] - whole[:n]) <= dc.HALF_STEP[dtype] * 4 * np.abs(whole).max())
    assert np.all(got[n:] == 5.0)
    x, q_out, k, v = put(gto, ctx, c)
    assert gto.gto_decode_status(ctx) == 8
    assert torch.all(q_out[n:] == 7.0) and (n == 0 or not torch.any((q_out[:n] == 7.0).all(-1)))
    verdict = dict(accept_len=torch.zeros(S, dtype=torch.int32, device=DEV), path_node=torch.zeros((S, 1), dtype=torch.int32, device=DEV),
                   token=torch.zeros((S, 2), dtype=torch.int32, device=DEV))
    new_len = torch.full((S,), -5, dtype=torch.int32, device=DEV)
    gto.gto_kv_commit(ctx, c.batch, verdict, k, v, new_len)
    assert new_len.tolist() == c.host["kv_len"][:at].tolist() + [-5] * (S - at)


# ------------------------------------------------------------------ what a step did not write is not kept

def small_step(gto, S=3, T=64, layers=2, g=0, max_pages=8):
    from paper_2509_22134_b200.runner import DecodeStep
    cfg = gto.make_decode_config(S=S, T=T, n_q_heads=4, n_kv_heads=2, head_dim=64, page_size=16, n_pages=S * max_pages,
                                 max_pages=max_pages, dtype="bf16", g=g, D=3, V_draft=64, V_target=64)
    step = DecodeStep(cfg, layers, FREQ, DEV)
    step.page_table.copy_(torch.arange(S * max_pages, dtype=torch.int32).view(S, max_pages))
    return step


def layers_of(step, tokens, seed=0):
    gen = torch.Generator(DEV).manual_seed(seed)
    for i in range(step.k_cache.shape[0]):
        x = torch.randn((tokens, 8, 64), generator=gen, device=DEV).to(torch.bfloat16)
        out = torch.zeros((tokens, 4, 64), dtype=torch.bfloat16, device=DEV)
        step.attend(i, x[:, :4], x[:, 4:6], x[:, 6:], out)


@pytest.mark.gpu
def test_a_chunk_behind_the_steps_tokens_is_not_committed(gto):
    """Sequence 2's chunk ends behind the rows that the layers were given, but within what the context takes."""
    step = small_step(gto)
    step.begin(torch.tensor([0, 5, 9, 20], dtype=torch.int32, device=DEV))
    layers_of(step, 12)
    step.commit()
    assert step.status() == 8
    assert step.kv_len.tolist() == [5, 4, 0]
    step.begin(torch.tensor([0, 1, 2, 13], dtype=torch.int32, device=DEV))   # and again, with all rows
    layers_of(step, 13)
    step.commit()
    assert step.status() == 0
    assert step.kv_len.tolist() == [6, 5, 11]


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,want", [(None, [13]), (13, [13]), (12, [-5]), (0, [-5])])
def test_commit_judges_a_batch_by_the_tokens_it_is_told(gto, tokens, want):
    c = dc.Case([13], [13], 4, 2, 64, 16, "bf16", seed=1, poison=0.0)
    verdict = dict(accept_len=torch.zeros(1, dtype=torch.int32, device=DEV), path_node=torch.zeros((1, 1), dtype=torch.int32, device=DEV),
                   token=torch.zeros((1, 2), dtype=torch.int32, device=DEV))
    new_len = torch.full((1,), -5, dtype=torch.int32, device=DEV)
    ctx = c.ctx(gto)
    gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, new_len, tokens=tokens)
    assert gto.gto_decode_status(ctx) == (0 if want == [13] else 8)
    assert new_len.tolist() == want
    for bad, error in ((-1, ValueError), (1 << 40, ValueError), (c.T + 1, gto.GtoError), ("x", TypeError)):
        with pytest.raises(error):
            gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, new_len, tokens=bad)


@pytest.mark.gpu
def test_a_chunk_without_its_page_is_not_committed(gto):
    """Append leaves out the tokens whose page the table does not name: the sequence's length may not count them."""
    step = small_step(gto)
    step.page_table[1, 1] = -1                                    # entries 16 .. 31 of sequence 1
    step.begin(torch.tensor([0, 5, 25, 30], dtype=torch.int32, device=DEV))
    layers_of(step, 30)
    assert step.status() == 8
    step.commit()
    assert step.status() == 8
    assert step.kv_len.tolist() == [5, 0, 5]
    step.page_table[1, 1] = 9
    step.begin(torch.tensor([0, 1, 21, 22], dtype=torch.int32, device=DEV))
    layers_of(step, 22)
    step.commit()
    assert step.status() == 0
    assert step.kv_len.tolist() == [6, 20, 6]


@pytest.mark.gpu
@pytest.mark.parametrize("missing,length,want", [(2, 0, 33), (2, 1, 34), (3, 0, 33), (3, 2, 35), (2, 2, -5), (1, 0, 33), (1, 1, 34)])
def test_commit_needs_the_pages_of_the_entries_that_stay_and_no_others(gto, missing, length, want):
    """A lead of 3 on 30 entries, in pages of 17: entries 30 .. 32 and the accepted nodes' 33, 34, ...; the tree reaches entry 53
    (page 3); page 2 begins at entry 34."""
    c = dc.Case([24], [54], 4, 2, 64, 17, "bf16", 21, 3, [21], seed=1, poison=0.0)
    if missing == 1:
        c.batch["page_table"][0, 0] = -1          # behind the chunk: attention needs it, commit does not
    else:
        c.batch["page_table"][0, missing] = -1
    path = [[0, -1, -1], [0, -1, -1], [0, 17, -1] if missing == 2 else [0, 1, -1]][length]
    verdict = dict(accept_len=torch.tensor([length], dtype=torch.int32, device=DEV),
                   path_node=torch.tensor([path], dtype=torch.int32, device=DEV), token=torch.zeros((1, 4), dtype=torch.int32, device=DEV))
    new_len = torch.full((1,), -5, dtype=torch.int32, device=DEV)
    ctx = c.ctx(gto)
    gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, new_len)
    assert new_len.tolist() == [want]
    assert gto.gto_decode_status(ctx) == (8 if want < 0 else 0)


@pytest.mark.gpu
def test_commit_skips_a_sequence_without_a_verdict(gto):
    """accept_len -1 is what gto_verify_tree leaves where a wait ran out; its path may hold anything."""
    c = dc.Case([7, 7, 7], [30, 40, 50], 4, 2, 64, 16, "bf16", 6, 3, seed=1, poison=0.0)
    ctx = c.ctx(gto)
    verdict = dict(accept_len=torch.tensor([-1, 1, 4], dtype=torch.int32, device=DEV),
                   path_node=torch.tensor([[0, 1, 2], [2, -1, -1], [0, 1, 2]], dtype=torch.int32, device=DEV),
                   token=torch.zeros((3, 4), dtype=torch.int32, device=DEV))
    k, v = c.dk.clone(), c.dv.clone()
    page, place = (int(x) for x in dec.slots(c.host, 1, 34, 16))
    to, at = (int(x) for x in dec.slots(c.host, 1, 36, 16))
    k[page, place], v[page, place] = c.dk[to, at], c.dv[to, at]
    new_len = torch.full((3,), -5, dtype=torch.int32, device=DEV)
    gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, new_len)
    assert gto.gto_decode_status(ctx) == 8
    assert new_len.tolist() == [-5, 35, -5]
    assert torch.equal(c.dk, k) and torch.equal(c.dv, v)


def test_the_header_names_every_call_whose_waits_can_run_out(repo_root):
    """The two kernels that raise the status bit belong to these calls."""
    import os
    import re
    src = os.path.join(repo_root, "paper_2509_22134_b200", "csrc")
    raising = {f for f in os.listdir(src) if f.endswith(".cu") and "atomicOr" in open(os.path.join(src, f)).read()
               and re.search(r"atomicOr\([^;]*kStatusTimeout", open(os.path.join(src, f)).read())}
    assert raising == {"tree_attention_tc.cu", "tree_verify.cu"}
    text = open(os.path.join(repo_root, "include", "gto.h")).read()
    entry = text[text.index("GTO_ERR_TIMEOUT = 6"):]
    entry = entry[:entry.index("*/")]
    assert "gto_tree_attention" in entry and "gto_verify_tree" in entry


# ------------------------------------------------------------------ outputs over what a call reads

def refused(gto, ctx, call):
    before = gto.gto_decode_launch_count(ctx)
    with pytest.raises(gto.GtoError) as e:
        call()
    assert e.value.code == 1 and gto.gto_decode_launch_count(ctx) == before


@pytest.mark.gpu
def test_commit_refuses_lengths_over_a_table_it_reads(gto):
    c = dc.Case([7, 7, 7], [30, 40, 50], 4, 2, 64, 16, "bf16", 6, 3, [6, 6, 6], seed=1, poison=0.0)
    ctx = c.ctx(gto)
    i32 = dict(dtype=torch.int32, device=DEV)
    verdict = dict(accept_len=torch.zeros(3, **i32), path_node=torch.zeros((3, 3), **i32), token=torch.zeros((3, 4), **i32))
    for over in (c.batch["kv_len"], c.batch["q_start"][:3], c.batch["q_start"][1:], c.batch["n_nodes"], verdict["accept_len"],
                 c.batch["page_table"].view(-1)[2:5], verdict["path_node"].view(-1)[4:7]):
        refused(gto, ctx, lambda: gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, over))
    gto.gto_kv_commit(ctx, c.batch, verdict, c.dk, c.dv, torch.zeros(3, **i32))
    assert gto.gto_decode_status(ctx) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_refuses_an_lse_over_queries_or_outputs(gto, dtype):
    c = dc.Case([7, 7], [30, 40], 4, 2, 64, 16, dtype, seed=1, poison=0.0)
    ctx = c.ctx(gto)
    out = torch.zeros_like(c.dq)
    for over in (c.dq, out):
        lse = over.view(-1).view(torch.float32)[:c.T * 4].view(c.T, 4)
        refused(gto, ctx, lambda: gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=lse))


@pytest.mark.gpu
def test_verify_refuses_a_verdict_over_what_it_reads(gto):
    cfg = gto.make_decode_config(S=3, g=6, D=3, V_draft=512, V_target=512, logit_dtype="f32")
    ctx = gto.gto_decode_create(cfg, 0)
    i32, f32 = dict(dtype=torch.int32, device=DEV), dict(device=DEV)
    tree = dict(node_token=torch.zeros((3, 6), **i32), node_parent=torch.full((3, 6), -1, **i32), n_nodes=torch.full((3,), 6, **i32))
    target, u = torch.zeros((3, 7, 512), **f32), torch.zeros((3, 6), **f32)
    temperature, bonus = torch.ones(3, **f32), torch.zeros(3, **f32)
    good = gto.alloc_verdict(cfg, DEV)
    call = lambda out: gto.gto_verify_tree(ctx, tree, target, None, temperature, u, bonus, out)
    as_i32 = lambda t, n: t.view(-1).view(torch.int32)[:n]
    for name, n, shape in (("accept_len", 3, (3,)), ("path_node", 9, (3, 3)), ("token", 12, (3, 4))):
        for over in (tree["node_token"], tree["node_parent"], tree["n_nodes"], target, u, temperature, bonus,
                     *(good[m] for m in good if m != name)):
            if over.numel() >= n:
                refused(gto, ctx, lambda: call({**good, name: as_i32(over, n).view(shape)}))
    call(good)
    assert gto.gto_decode_status(ctx) == 0


@pytest.mark.gpu
def test_an_array_without_elements_lies_over_nothing(gto):
    """Without trees the node arrays have no elements: where they point does not matter."""
    import ctypes
    cfg = gto.make_decode_config(S=2, g=0, D=1, V_draft=64, V_target=64, logit_dtype="f32")
    ctx = gto.gto_decode_create(cfg, 0)
    out = gto.alloc_verdict(cfg, DEV)
    buf = torch.zeros(4, dtype=torch.int32, device=DEV)
    target, t, u = torch.zeros((2, 1, 64), device=DEV), torch.zeros(2, device=DEV), torch.zeros(2, device=DEV)
    tree = gto.gto_draft_tree(2, buf.data_ptr() + 4, buf.data_ptr() + 4, None, None, None)
    verdict = gto.gto_verdict(buf.data_ptr(), out["path_node"].data_ptr(), out["token"].data_ptr())
    code = gto._lib.gto_verify_tree(ctypes.c_void_p(ctx.handle), ctypes.byref(tree), ctypes.c_void_p(target.data_ptr()), None,
                                    ctypes.c_void_p(t.data_ptr()), ctypes.c_void_p(buf.data_ptr() + 4), ctypes.c_void_p(u.data_ptr()),
                                    ctypes.byref(verdict), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert code == 0 and gto.gto_decode_status(ctx) == 0
    assert buf[:2].tolist() == [0, 0] and out["token"][:, 0].tolist() == [0, 0]
