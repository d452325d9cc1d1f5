"""How exact the decoding step's attention is, on inputs where a coarser kernel would pass for a right one."""
import numpy as np
import pytest
import torch

import decode_cases as dc
from oracle import decode_oracle as dec

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,gap", [(60001, 17.6), (60001, 17.156), (300001, 17.6), (5000, 9.0)])
def test_a_flat_tail_behind_one_large_score_is_kept(gto, n, gap, dh, dtype):
    """One entry, of value 0, has a score `gap` above all others, which are equal: each of them weighs about 2^-25 of it
    and together they are the whole output.  As many sequences as make every SM go through whole rows read one cache.

    Tolerance.  The tail's weights are equal, so their roundings are too: half a step, relative to a weight as long as the
    type holds it as a normal number (fp16: down to 2^-25 of the row's largest; 17.6 is 2^-25.4 of it, where a step is
    2^0.4 times as large against the weight), and the output is rounded once: 2.4 half steps, 3 are allowed.  The score is a
    product of two numbers and its scale is 1: both exact; exp in fp32: 2^-18 covers 2^-22 for a weight and 2^-24 |score| for
    its argument.  Sums of equal terms err the same way at every step: a row's tiles of 64 go to two streams, `tiles`
    each; the fp32 sum of the weights rounds once a tile, the output's accumulator four times and may cut (2^-23), both on a
    sum that is half of the last one on the average."""
    S, page = 160, 128
    pages = -(-n // page)
    k = torch.zeros((pages, page, 1, dh), dtype=torch.float64)
    gen = torch.Generator().manual_seed(n + dh)
    v = (1 + 0.25 * torch.randn(k.shape, generator=gen)).to(dc.TORCH[dtype])
    k[0, 0, 0, 0] = gap / 8
    v[0, 0] = 0
    k = k.to(dc.TORCH[dtype])
    top = float(k[0, 0, 0, 0]) * 8
    w = np.exp(-top)
    want = w * v.view(-1, dh)[:n].double().sum(0) / (1 + w * (n - 1))
    q = torch.zeros((S, 1, dh), dtype=dc.TORCH[dtype], device=DEV)
    q[:, :, 0] = 8
    batch = dict(q_start=torch.arange(S + 1, dtype=torch.int32, device=DEV), kv_len=torch.full((S,), n, dtype=torch.int32, device=DEV),
                 page_table=torch.arange(pages, dtype=torch.int32, device=DEV).repeat(S, 1))
    cfg = gto.make_decode_config(S=S, T=S, n_q_heads=1, n_kv_heads=1, head_dim=dh, page_size=page, n_pages=pages, max_pages=pages,
                                 dtype=dtype, softmax_scale=1.0)
    ctx = gto.gto_decode_create(cfg, 0)
    out, lse = torch.zeros_like(q), torch.zeros((S, 1), device=DEV)
    gto.gto_tree_attention(ctx, batch, q, k.to(DEV), v.to(DEV), out, lse=lse)
    assert gto.gto_decode_status(ctx) == 0
    tiles = n / 128 + 1
    err = (out.double().cpu()[:, 0] - want).abs()
    assert torch.all(err <= want * (3 * dc.HALF_STEP[dtype] + 2.0 ** -18 + 4 * tiles * 2.0 ** -24)), float((err / want).max())
    err = (lse.double().cpu() - (top + np.log1p(w * (n - 1)))).abs()
    assert torch.all(err <= 2.0 ** -18 + tiles * 2.0 ** -25 + 2.0 ** -22 * top), float(err.max())


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("q_lens,kv_lens,g,hq,dh", [
    ([13], [70], 12, 4, 64),                     # one block, both streams on its tiles
    ([13], [4000], 12, 8, 128),                  # cut into many parts
    ([13] * 40, [1500] * 40, 12, 8, 64),
    ([129], [300], 128, 8, 128),                 # two row tiles, two words of a mask
    ([70], [90], 0, 16, 64),                     # a prompt
])
def test_a_value_that_is_not_finite_spoils_no_lse_and_no_row_that_does_not_see_it(gto, q_lens, kv_lens, g, hq, dh, bad, dtype):
    c = dc.Case(q_lens, kv_lens, hq, 2, dh, 16, dtype, g, 5, seed=len(q_lens) + g, poison=0.0)
    scale = dh ** -0.5
    want, want_z, spread = c.attention_on_device(scale)
    sees = np.zeros(c.T, bool)
    for s in range(c.S):
        n, L = q_lens[s], kv_lens[s]
        hit = 5 if g else n - 20                               # entry L - n + lead + 5, or the prompt's 20th from its end
        e = L - g + hit if g else L - n + hit
        page, place = dec.slots(c.host, s, [e], c.page)
        c.v[page, place] = bad
        q0 = int(c.host["q_start"][s])
        if g:
            sees[q0 + n - g:q0 + n] = c.host["node_mask"][s][:, hit]
        else:
            sees[q0 + hit:q0 + n] = True
    c.dv = c.pool(c.v)
    ctx = c.ctx(gto, softmax_scale=scale)
    out, lse = torch.zeros_like(c.dq), torch.zeros((c.T, hq), device=DEV)
    gto.gto_tree_attention(ctx, c.batch, c.dq, c.dk, c.dv, out, lse=lse)
    assert gto.gto_decode_status(ctx) == 0
    got, z = out.double().cpu().numpy()[:c.n], lse.double().cpu().numpy()[:c.n]
    assert np.all(np.abs(z - want_z[:c.n]) <= 1e-4)             # dh products of at most about 10 in fp32: 128 * 10 * 2^-23 / 11
    blind = ~sees[:c.n]
    assert np.all(np.abs(got[blind] - want[:c.n][blind]) <= spread[:c.n][blind] * (dc.HALF_STEP[dtype] * 2 + 1e-3))
    assert not np.isfinite(got[sees[:c.n]]).any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("low", [23265282, 9000000, 726815, 1000])
def test_scores_whose_exponents_fp32_knows_roughly_give_finite_weights(gto, low, dtype):
    """Scores of `low` and a little more in later tiles, where fp32 numbers are up to 4 apart: the weight of an exponent
    rounded up, relative to a reference below the maximum, could pass what fp16 holds.  All values are 1.5, so that the output
    is 1.5 whatever the weights are, if they are finite: each is rounded (half a step), their sum is not, and the result once.
    A score is unit a + b, all of them numbers of the type: exact in fp32."""
    S, n, dh = 300, 500, 64
    bits = 2 ** 11 if dtype == "f16" else 2 ** 8
    k = torch.zeros((-(-n // 16), 16, 1, dh), dtype=torch.float64)
    flat = k.view(-1, dh)
    unit = 512 if low > 2 ** 24 else 256
    a = low // unit
    a -= a % max(1, 2 ** max(0, int(a).bit_length() - int(bits).bit_length() + 1))      # (a number that the type holds)
    b = min(low - unit * a, 200)
    for tile, more in enumerate([0, 2, 2, 6, 4, 2, 2]):
        flat[tile * 64 + 7, 0] = a
        flat[tile * 64 + 7, 1] = b + more
    k, v = k.to(dc.TORCH[dtype]), torch.full_like(k, 1.5).to(dc.TORCH[dtype])
    assert k[0, 7, 0, 0] == a
    q = torch.zeros((S, 1, dh), dtype=dc.TORCH[dtype], device=DEV)
    q[:, :, 0], q[:, :, 1] = unit, 1
    batch = dict(q_start=torch.arange(S + 1, dtype=torch.int32, device=DEV), kv_len=torch.full((S,), n, dtype=torch.int32, device=DEV),
                 page_table=torch.arange(k.shape[0], dtype=torch.int32, device=DEV).repeat(S, 1))
    cfg = gto.make_decode_config(S=S, T=S, n_q_heads=1, n_kv_heads=1, head_dim=dh, page_size=16, n_pages=k.shape[0],
                                 max_pages=k.shape[0], dtype=dtype, softmax_scale=1.0)
    ctx = gto.gto_decode_create(cfg, 0)
    out, lse = torch.zeros_like(q), torch.zeros((S, 1), device=DEV)
    gto.gto_tree_attention(ctx, batch, q, k.to(DEV), v.to(DEV), out, lse=lse)
    assert gto.gto_decode_status(ctx) == 0
    assert torch.all((out.double() - 1.5).abs() <= 1.5 * (2 * dc.HALF_STEP[dtype] + 2.0 ** -20))
    x = torch.from_numpy(float(unit * a + b) + np.array([0, 2, 2, 6, 4, 2, 2.0]))
    assert torch.all((lse.double() - torch.logsumexp(x, 0)).abs() <= 2.0 ** -22 * x[0] + 2.0 ** -18)
