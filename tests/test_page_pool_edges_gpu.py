"""The page calls where their documentation ends: pools without sequences, broken names, contexts without pages."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


def make(gto, S=4, n_pages=12, max_pages=5, page=4, layers=2):
    cfg = gto.make_decode_config(S=S, T=S, n_q_heads=1, n_kv_heads=1, head_dim=16, page_size=page, n_pages=n_pages, max_pages=max_pages,
                                 dtype="f32", flags=gto.GTO_DECODE_PAGES)
    k, v = (torch.randn((layers, n_pages, page, 1, 16), device=DEV) for _ in range(2))
    return gto.gto_decode_create(cfg, 0), cfg, k, v


@pytest.mark.parametrize("counts", [[0] * 12, [0, 2, 0, 0, 1, 0, 0, 1, 0, 0, 0, 3]])
def test_compact_of_a_pool_without_sequences(gto, counts):
    """The counts alone decide (whoever holds the pages); every output is written."""
    ctx, cfg, k, v = make(gto)
    pool = gto.alloc_page_pool(cfg, DEV, 0)
    pool["ref_count"].copy_(torch.tensor(counts))
    table, ref, used = torch.full((0, 5), -9, **I32), torch.full((12,), -9, **I32), torch.full((1,), -9, **I32)
    was = k.clone(), v.clone()
    gto.gto_pages_compact(ctx, pool, k, v, table, ref, used)
    assert gto.gto_decode_status(ctx) == 0
    n = sum(c > 0 for c in counts)
    assert used.item() == n
    moves = list(zip([p for p in range(n, 12) if counts[p]], [p for p in range(n) if not counts[p]]))
    want = [counts[p] if p < n else 0 for p in range(12)]
    for x, y in zip((k, v), was):
        for a, b in moves:
            y[:, b] = y[:, a]
            want[b] = counts[a]
        assert torch.equal(x, y)
    assert ref.tolist() == want and pool["ref_count"].tolist() == counts


def test_compact_of_a_pool_without_sequences_refuses_what_it_would_write_over(gto):
    ctx, cfg, k, v = make(gto)
    pool = gto.alloc_page_pool(cfg, DEV, 0)
    table, ref, used = torch.zeros((0, 5), **I32), torch.zeros(12, **I32), torch.zeros(1, **I32)
    for bad in (dict(ref=pool["ref_count"]), dict(used=pool["ref_count"][:1]), dict(used=ref[3:4])):
        args = dict(ref=ref, used=used) | bad
        with pytest.raises(gto.GtoError) as e:
            gto.gto_pages_compact(ctx, pool, k, v, table, args["ref"], args["used"])
        assert e.value.code == 1
    inside = torch.zeros((3, 5), **I32)
    gto.gto_pages_compact(ctx, pool, k, v, inside[1:1], ref, used)  # nothing lies over anything
    assert gto.gto_decode_status(ctx) == 0
