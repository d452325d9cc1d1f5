"""What gto_sample_tokens, gto_verify_tree_limited and the page calls refuse."""
import pytest
import torch

CACHE = dict(S=4, T=16, n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, n_pages=10, max_pages=5, dtype="bf16")
ROWS = dict(S=4, g=3, D=2, V_draft=512, V_target=512, logit_dtype="bf16")


@pytest.mark.parametrize("kw,code", [
    (dict(ROWS, flags=4), 1),                                           # pages without a cache
    (dict(CACHE, flags=8), 1),
    (dict(CACHE, flags=4, S=1 << 20, max_pages=1 << 14), 2),            # a copy of the table would have 64 GB
    (dict(CACHE, flags=4, S=1 << 16, max_pages=1 << 15), 2),            # slots are counted in 32 bits
    (dict(CACHE, flags=4, n_pages=(1 << 30) + 1), 2),
])
def test_configurations_are_refused_without_a_device(kw, code):
    from paper_2509_22134_b200 import binding as gto
    with pytest.raises(gto.GtoError) as e:
        gto.gto_decode_create(gto.make_decode_config(**kw), 0)
    assert e.value.code == code


def test_struct_layouts_match_the_header(repo_root):
    import os
    import re
    from paper_2509_22134_b200 import binding as gto
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(repo_root, "include", "gto.h")).read(), flags=re.S)
    for struct in (gto.gto_limits, gto.gto_page_pool):
        end = text.index("} %s;" % struct.__name__)
        body = text[text.rindex("typedef struct {", 0, end) + 16:end]
        names = [re.sub(r"\W", "", re.sub(r"^(const\s+)?\w+", "", line.strip())) for line in body.split(";") if line.strip()]
        assert names == [f[0] for f in struct._fields_], struct.__name__
    assert "pages" in gto.gto_status_string(9)


def test_a_null_context_is_refused():
    import ctypes
    from paper_2509_22134_b200 import binding as gto
    lib, zero = ctypes.CDLL(gto.LIB_PATH), ctypes.c_void_p(None)
    assert lib.gto_sample_tokens(zero, zero, ctypes.c_int64(8), 1, zero, 1, zero, zero, zero, zero, zero, zero) == 1
    assert lib.gto_verify_tree_limited(*[zero] * 9) == 1
    assert lib.gto_pages_fork(*[zero] * 4) == lib.gto_pages_resize(*[zero] * 5) == lib.gto_pages_compact(*[zero] * 7) == 1


# ------------------------------------------------------------------ with a device

F32, I32 = dict(device="cuda:0"), dict(dtype=torch.int32, device="cuda:0")


@pytest.mark.gpu
def test_sample_refuses_wrong_arguments():
    from paper_2509_22134_b200 import binding as gto
    ctx = gto.gto_decode_create(gto.make_decode_config(**ROWS), 0)
    z = torch.zeros((3, 512), dtype=torch.bfloat16, device="cuda:0")
    good = dict(logits=z, limits=dict(temperature=torch.ones(3, **F32)), u=torch.zeros(3, **F32), token=torch.zeros(3, **I32),
                logp=torch.zeros(3, **F32), n_kept=torch.zeros(3, **I32), rows=None)

    def call(**kw):
        a = dict(good, **kw)
        gto.gto_sample_tokens(ctx, a["logits"], a["limits"], a["u"], a["token"], logp=a["logp"], n_kept=a["n_kept"], rows=a["rows"])

    call()
    call(logp=None, n_kept=None)
    heat = good["limits"]["temperature"]
    for kw in (dict(logits=z.float()), dict(logits=z[:, :504]), dict(logits=z[:2]), dict(logits=z.cpu()), dict(logits=z.t()),
               dict(logits=z[0]), dict(limits=None), dict(limits=dict(temperature=heat.double())), dict(limits=dict(temperature=1.0)),
               dict(limits=dict(temperature=heat, top_k=torch.zeros(3, **F32))), dict(limits=dict(temperature=heat, top_p=torch.zeros(2, **F32))),
               dict(limits=dict(temperature=heat, min_p=torch.zeros(3, **I32))), dict(u=torch.zeros(4, **F32)), dict(u=None),
               dict(token=torch.zeros(3, dtype=torch.int64, device="cuda:0")), dict(logp=torch.zeros(2, **F32)),
               dict(n_kept=torch.zeros(3, **F32)), dict(rows=torch.zeros(2, **I32)), dict(rows=torch.zeros(3, **F32))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(KeyError):
        call(limits=dict(top_p=heat))
    shared = torch.zeros(4, **I32)
    odd = torch.zeros(2000, dtype=torch.bfloat16, device="cuda:0")
    five = dict(limits=dict(temperature=torch.ones(5, **F32)), u=torch.zeros(5, **F32), token=torch.zeros(5, **I32), logp=None, n_kept=None,
                logits=torch.zeros((5, 512), dtype=torch.bfloat16, device="cuda:0"))
    for kw in (five,                                                      # more than the context takes
               dict(token=shared[:3], n_kept=shared[1:]),                  # outputs over each other
               dict(logp=heat), dict(logp=good["u"]),                      # and over what is read
               dict(token=shared[:3], rows=shared[1:]),
               dict(logits=odd[4:4 + 1536].view(3, 512)),                  # rows that do not start on 16 bytes
               dict(logits=odd[:1548].as_strided((3, 512), (516, 1)))):
        with pytest.raises(gto.GtoError) as e:
            call(**kw)
        assert e.value.code == 1
    call(rows=torch.zeros(3, **I32), logits=z[:1])
    assert gto.gto_decode_status(ctx) == 0
    none = {k: (v[:0] if torch.is_tensor(v) else v) for k, v in good.items()}
    none["limits"] = dict(temperature=heat[:0])
    n = gto.gto_decode_launch_count(ctx)
    call(**none)
    assert gto.gto_decode_launch_count(ctx) == n                          # nobody to draw for
    pages = gto.gto_decode_create(gto.make_decode_config(**CACHE), 0)
    with pytest.raises((ValueError, gto.GtoError)):
        gto.gto_sample_tokens(pages, z[:, :0], good["limits"], good["u"], good["token"])


@pytest.mark.gpu
def test_verify_limited_refuses_wrong_arguments():
    from paper_2509_22134_b200 import binding as gto
    ctx = gto.gto_decode_create(gto.make_decode_config(**ROWS), 0)
    tree = dict(node_token=torch.zeros((2, 3), **I32), node_parent=torch.full((2, 3), -1, **I32))
    target = torch.zeros((2, 4, 512), dtype=torch.bfloat16, device="cuda:0")
    out = gto.alloc_verdict(ctx.cfg, "cuda:0", 2)
    limits = dict(temperature=torch.ones(2, **F32), top_p=torch.ones(2, **F32))
    args = [tree, target, None, limits, torch.zeros((2, 3), **F32), torch.zeros(2, **F32), out]
    gto.gto_verify_tree_limited(ctx, *args)
    for i, bad in ((0, None), (1, target[:, :3].contiguous()), (1, target.float()), (2, torch.zeros(512, device="cuda:0")), (3, limits["top_p"]),
                   (3, dict(limits, top_k=torch.zeros(2, **F32))), (4, torch.zeros((2, 2), **F32)), (5, torch.zeros(3, **F32)),
                   (6, gto.alloc_verdict(ctx.cfg, "cuda:0", 3))):
        with pytest.raises(ValueError):
            gto.gto_verify_tree_limited(ctx, *(args[:i] + [bad] + args[i + 1:]))
    for bad in (dict(out, accept_len=limits["top_p"].view(torch.int32)), dict(out, token=tree["node_token"].view(-1)[:6].view(2, 3))):
        with pytest.raises(gto.GtoError) as e:                            # outputs over what is read
            gto.gto_verify_tree_limited(ctx, *(args[:6] + [bad]))
        assert e.value.code == 1
    assert gto.gto_decode_status(ctx) == 0


@pytest.mark.gpu
def test_page_calls_refuse_wrong_arguments():
    from paper_2509_22134_b200 import binding as gto
    cfg = gto.make_decode_config(**CACHE, flags=gto.GTO_DECODE_PAGES)
    ctx = gto.gto_decode_create(cfg, 0)
    pool = gto.alloc_page_pool(cfg, "cuda:0")
    k, v = (torch.zeros((2, 10, 16, 2, 64), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    n = torch.zeros(4, **I32)
    t, r, m = torch.zeros((4, 5), **I32), torch.zeros(10, **I32), torch.zeros(1, **I32)
    fork = lambda pool=pool, n=n, ctx=ctx: gto.gto_pages_fork(ctx, pool, n)
    resize = lambda pool=pool, n=n, k=k, v=v, ctx=ctx: gto.gto_pages_resize(ctx, pool, n, k, v)
    compact = lambda pool=pool, k=k, t=t, r=r, m=m, ctx=ctx: gto.gto_pages_compact(ctx, pool, k, v, t, r, m)
    fork(), resize(), compact()
    for call in (fork, resize, compact):
        for bad in (None, dict(pool, held=pool["held"][:3]), dict(pool, page_table=pool["page_table"][:, :4]),
                    dict(pool, ref_count=pool["ref_count"].long()), dict(pool, kv_len=pool["kv_len"].cpu())):
            with pytest.raises(ValueError):
                call(pool=bad)
        with pytest.raises(KeyError):
            call(pool={n: x for n, x in pool.items() if n != "ref_count"})
        with pytest.raises(gto.GtoError) as e:
            call(pool=dict(pool, held=pool["kv_len"]))                    # two tables in one place
        assert e.value.code == 1
        with pytest.raises(gto.GtoError) as e:                            # a context without the workspace
            call(ctx=gto.gto_decode_create(gto.make_decode_config(**CACHE), 0))
        assert e.value.code == 1
        big = gto.alloc_page_pool(cfg, "cuda:0", 5)
        with pytest.raises((gto.GtoError, ValueError)):                   # more sequences than the context takes
            call(pool=big)
    for call in (fork, resize):
        for bad in (n[:3], n.float(), n.cpu()):
            with pytest.raises(ValueError):
                call(n=bad)
        with pytest.raises(gto.GtoError) as e:
            call(n=pool["kv_len"])
        assert e.value.code == 1
    for bad in (k[:, :9], k.float(), k[0, 0]):
        with pytest.raises(ValueError):
            resize(k=bad)
        with pytest.raises(ValueError):
            compact(k=bad)
    for kw in (dict(t=pool["page_table"]), dict(r=pool["ref_count"]), dict(m=r[:1]), dict(m=pool["held"][:1])):
        with pytest.raises(gto.GtoError) as e:
            compact(**kw)
        assert e.value.code == 1
    for kw in (dict(t=t[:, :4]), dict(r=r[:9]), dict(m=m.long())):
        with pytest.raises(ValueError):
            compact(**kw)
    none = gto.alloc_page_pool(cfg, "cuda:0", 0)
    count = gto.gto_decode_launch_count(ctx)
    fork(pool=none, n=n[:0]), resize(pool=none, n=n[:0])
    assert gto.gto_decode_launch_count(ctx) == count and gto.gto_decode_status(ctx) == 0
