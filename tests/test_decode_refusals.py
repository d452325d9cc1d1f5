"""What the decoding-step calls refuse: configurations (on the CPU) and call arguments (a context needs a device)."""
import pytest
import torch

GOOD = dict(S=4, T=16, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_pages=4, dtype="bf16", g=12, D=3,
            V_draft=512, V_target=512, logit_dtype="bf16")


@pytest.mark.parametrize("kw,code", [
    (dict(S=0), 1), (dict(T=-1), 1), (dict(g=-1), 1), (dict(D=0), 1), (dict(n_q_heads=7), 1), (dict(n_q_heads=0), 1),
    (dict(head_dim=0, softmax_scale=1.0), 1), (dict(page_size=0), 1), (dict(n_pages=0), 1), (dict(max_pages=0), 1),
    (dict(rope_dims=80), 1), (dict(softmax_scale=0.0), 1), (dict(softmax_scale=float("nan")), 1), (dict(softmax_scale=float("inf")), 1),
    (dict(norm_eps=-1.0), 1), (dict(V_draft=513, V_target=512), 1), (dict(V_draft=8, V_target=512), 1), (dict(flags=64), 1),
    (dict(flags=2), 1),                                      # context rows without k
    (dict(n_kv_heads=0, n_q_heads=0, V_target=0), 1),        # neither cache nor verification
    (dict(g=129), 2), (dict(D=17), 2), (dict(head_dim=72), 2), (dict(head_dim=272), 2), (dict(rope_dims=24), 2),
    (dict(n_q_heads=258), 2), (dict(max_pages=1 << 27), 2), (dict(T=1 << 28), 2),
    (dict(V_draft=512, V_target=1001), 2), (dict(V_target=1 << 20), 2), (dict(flags=2, k=17), 2),
])
def test_configurations_are_refused_without_a_device(kw, code):
    from paper_2509_22134_b200 import binding as gto
    with pytest.raises(gto.GtoError) as e:
        gto.gto_decode_create(gto.make_decode_config(**dict(GOOD, **kw)), 0)
    assert e.value.code == code


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a device only")
def test_a_good_configuration_needs_a_device():
    from paper_2509_22134_b200 import binding as gto
    with pytest.raises(gto.GtoError) as e:
        gto.gto_decode_create(gto.make_decode_config(**GOOD), 0)
    assert e.value.code == 4


def test_struct_layouts_match_the_header(repo_root):
    import os
    import re
    from paper_2509_22134_b200 import binding as gto
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(repo_root, "include", "gto.h")).read(), flags=re.S)
    for struct in (gto.gto_decode_config, gto.gto_batch, gto.gto_kv_cache, gto.gto_draft_tree, gto.gto_verdict):
        end = text.index("} %s;" % struct.__name__)
        body = text[text.rindex("typedef struct {", 0, end) + 16:end]
        names = []
        for line in body.split(";"):
            line = line.strip()
            if line:
                decl = re.sub(r"^(const\s+)?\w+", "", line)
                names += [re.sub(r"\W", "", part) for part in decl.split(",")]
        assert names == [f[0] for f in struct._fields_], struct.__name__


# ------------------------------------------------------------------ with a device

@pytest.fixture
def made():
    from paper_2509_22134_b200 import binding as gto
    ctx = gto.gto_decode_create(gto.make_decode_config(**GOOD), 0)
    i32 = dict(dtype=torch.int32, device="cuda:0")
    batch = dict(q_start=torch.tensor([0, 13], **i32), kv_len=torch.tensor([20], **i32), page_table=torch.zeros((1, 4), **i32),
                 node_mask=torch.ones((1, 12, 1), dtype=torch.int64, device="cuda:0"), node_depth=torch.ones((1, 12), **i32))
    bf = dict(dtype=torch.bfloat16, device="cuda:0")
    t = dict(q=torch.zeros((16, 8, 64), **bf), k=torch.zeros((16, 2, 64), **bf), v=torch.zeros((16, 2, 64), **bf),
             out=torch.zeros((16, 8, 64), **bf), kc=torch.zeros((10, 16, 2, 64), **bf), vc=torch.zeros((10, 16, 2, 64), **bf),
             f=torch.zeros(32, dtype=torch.float64, device="cuda:0"))
    return gto, ctx, batch, t


def attention(m, batch=None, **kw):
    gto, ctx, b, t = m
    t = dict(t, **kw)
    gto.gto_tree_attention(ctx, batch or b, t["q"], t["kc"], t["vc"], t["out"])


def append(m, batch=None, **kw):
    gto, ctx, b, t = m
    t = {**t, "qn": None, **kw}
    gto.gto_kv_append(ctx, batch or b, t["q"], t["k"], t["v"], t["out"], t["kc"], t["vc"], t["f"], q_norm=t["qn"])


@pytest.mark.gpu
@pytest.mark.parametrize("change", [
    lambda t: dict(q=t["q"].float()), lambda t: dict(q=t["q"][:, :4]), lambda t: dict(q=t["q"].cpu()),
    lambda t: dict(q=t["q"].transpose(0, 1)), lambda t: dict(out=t["out"][:, ::2]), lambda t: dict(kc=t["kc"][:5]),
    lambda t: dict(kc=t["kc"].transpose(-1, -2)), lambda t: dict(kc=t["kc"].float()), lambda t: dict(vc=t["vc"][None]),
])
def test_attention_refuses_wrong_tensors(made, change):
    attention(made)
    with pytest.raises(ValueError):
        attention(made, **change(made[3]))


@pytest.mark.gpu
def test_calls_refuse_wrong_batches_and_overlaps(made):
    gto, ctx, b, t = made
    i32 = dict(dtype=torch.int32, device="cuda:0")
    many = dict(b, q_start=torch.zeros(6, **i32), kv_len=torch.zeros(5, **i32), page_table=torch.zeros((5, 4), **i32),
                node_mask=None, node_depth=None)
    for call in (attention, append):
        with pytest.raises(gto.GtoError) as e:
            call(made, batch=many)                           # more sequences than the context takes
        assert e.value.code == 1
        with pytest.raises(ValueError):
            call(made, batch=dict(b, kv_len=b["kv_len"].long()))
        with pytest.raises(ValueError):
            call(made, batch=dict(b, page_table=b["page_table"][:, :3]))
    for gone, call in (("node_mask", attention), ("node_depth", append)):
        with pytest.raises(gto.GtoError) as e:               # a tree without what the call reads of it
            call(made, batch={k: v for k, v in b.items() if k != gone})
        assert e.value.code == 1
    with pytest.raises(gto.GtoError) as e:                   # sizes of trees without trees
        attention(made, batch=dict(q_start=b["q_start"], kv_len=b["kv_len"], page_table=b["page_table"], n_nodes=torch.zeros(1, **i32)))
    assert e.value.code == 1
    with pytest.raises(gto.GtoError) as e:
        attention(made, out=t["q"])                          # out over q
    assert e.value.code == 1
    big = torch.zeros((17, 8, 64), dtype=torch.bfloat16, device="cuda:0")
    with pytest.raises(gto.GtoError) as e:
        attention(made, q=big, out=torch.zeros_like(big))    # more tokens than the context takes
    assert e.value.code == 1
    qkv = torch.zeros((16, 12, 64), dtype=torch.bfloat16, device="cuda:0")
    flat = qkv.view(-1)
    with pytest.raises(gto.GtoError) as e:                   # rotated queries over the projection they come from
        append(made, q=qkv[:, :8], out=flat[:16 * 8 * 64].view(16, 8, 64))
    assert e.value.code == 1
    with pytest.raises(gto.GtoError) as e:                   # a row that does not start on 16 bytes
        append(made, k=torch.zeros(16 * 128 + 4, dtype=torch.bfloat16, device="cuda:0")[4:].view(16, 2, 64))
    assert e.value.code == 1
    with pytest.raises(ValueError):
        append(made, f=t["f"].float())
    with pytest.raises(ValueError):
        append(made, qn=torch.ones(32, dtype=torch.bfloat16, device="cuda:0"))
    verdict = dict(accept_len=torch.zeros(1, **i32), path_node=torch.zeros((1, 3), **i32), token=torch.zeros((1, 4), **i32))
    with pytest.raises(gto.GtoError) as e:                   # the new lengths over the old ones
        gto.gto_kv_commit(ctx, b, verdict, t["kc"], t["vc"], b["kv_len"])
    assert e.value.code == 1
    assert gto.gto_decode_status(ctx) == 0 and gto.gto_decode_launch_count(ctx) == 0


@pytest.mark.gpu
def test_verify_refuses_wrong_arguments(made):
    gto, ctx, b, t = made
    i32 = dict(dtype=torch.int32, device="cuda:0")
    f32 = dict(device="cuda:0")
    tree = dict(node_token=torch.zeros((2, 12), **i32), node_parent=torch.full((2, 12), -1, **i32))
    target = torch.zeros((2, 13, 512), dtype=torch.bfloat16, device="cuda:0")
    out = gto.alloc_verdict(ctx.cfg, "cuda:0", 2)
    args = [tree, target, None, torch.ones(2, **f32), torch.zeros((2, 12), **f32), torch.zeros(2, **f32), out]
    for i, bad in ((1, target[:, :12].contiguous()), (1, target.float()), (2, torch.zeros(512, device="cuda:0")),
                   (3, torch.ones(2, dtype=torch.float64, device="cuda:0")), (4, torch.zeros((2, 11), **f32)),
                   (5, torch.zeros(3, **f32)), (6, gto.alloc_verdict(ctx.cfg, "cuda:0", 3))):
        with pytest.raises(ValueError):
            gto.gto_verify_tree(ctx, *(args[:i] + [bad] + args[i + 1:]))
    small = gto.gto_decode_create(gto.make_decode_config(S=2, g=12, D=3, V_draft=256, V_target=512), 0)
    with pytest.raises(gto.GtoError) as e:                   # a reduced vocabulary without its map
        gto.gto_verify_tree(small, *args)
    assert e.value.code == 1
