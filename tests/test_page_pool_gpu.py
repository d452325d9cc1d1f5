"""gto_pages_fork, gto_pages_resize and gto_pages_compact against the oracle: tables, counts and every byte of the cache."""
import numpy as np
import pytest
import torch

from oracle import pages_oracle as pg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def gto():
    from paper_2509_22134_b200 import binding
    return binding


class Pool:
    """The same pool on the host and on the device."""

    def __init__(self, gto, S, width, n_pages, page=4, layers=2, hkv=2, dh=16, dtype="f32", order="entry", seed=0):
        self.gto, self.page, self.S, self.width, self.n_pages = gto, page, S, width, n_pages
        cfg = gto.make_decode_config(S=S, T=S, n_q_heads=hkv, n_kv_heads=hkv, head_dim=dh, page_size=page, n_pages=n_pages,
                                     max_pages=width, dtype=dtype, flags=gto.GTO_DECODE_PAGES)
        self.ctx = gto.gto_decode_create(cfg, 0)
        self.dev = gto.alloc_page_pool(cfg, DEV)
        self.host = {k: v.cpu().numpy() for k, v in self.dev.items()}
        gen = torch.Generator(DEV).manual_seed(seed)
        make = {"entry": lambda: torch.randn((layers, n_pages, page, hkv, dh), generator=gen, device=DEV),
                "head": lambda: torch.randn((layers, n_pages, hkv, page, dh), generator=gen, device=DEV).transpose(2, 3),
                "page": lambda: torch.randn((n_pages, layers, page, hkv, dh), generator=gen, device=DEV).transpose(0, 1),
                "gaps": lambda: torch.randn((layers, n_pages, page, hkv + 1, 2 * dh), generator=gen, device=DEV)[:, :, :, :hkv, :dh]}
        keep = lambda t: torch.empty_strided(t.size(), t.stride(), dtype=TORCH[dtype], device=DEV).copy_(t)
        self.k, self.v = keep(make[order]()), keep(make[order]())
        self.hk, self.hv = self.k.clone(), self.v.clone()

    def put(self):
        for n, v in self.host.items():
            self.dev[n].copy_(torch.from_numpy(v.astype(np.int32)))

    def compare(self, status=0):
        assert self.gto.gto_decode_status(self.ctx) == status
        for n, v in self.host.items():
            assert np.array_equal(self.dev[n].cpu().numpy(), v), n
        assert torch.equal(self.k, self.hk) and torch.equal(self.v, self.hv)

    def fork(self, parent, stream=None):
        parent = np.asarray(parent, np.int32)
        self.host, bad = pg.fork(self.host, parent, self.page)
        self.gto.gto_pages_fork(self.ctx, self.dev, torch.from_numpy(parent).to(DEV), stream=stream)
        self.compare(8 if bad else 0)

    def resize(self, want, expect=None):
        want = np.asarray(want, np.int32)
        self.host, copies, bad, short = pg.resize(self.host, want, self.page)
        for a, b, n in copies:
            for x in (self.hk, self.hv):
                x[:, b, :n] = x[:, a, :n]
        self.gto.gto_pages_resize(self.ctx, self.dev, torch.from_numpy(want).to(DEV), self.k, self.v)
        self.compare(8 if bad else 9 if short else 0)
        return copies

    def compact(self, take=True):
        table, counts, used, moves = pg.compact(self.host)
        t, r, n = torch.full_like(self.dev["page_table"], -9), torch.full_like(self.dev["ref_count"], -9), torch.zeros(1, dtype=torch.int32, device=DEV)
        for a, b in moves:
            self.hk[:, b], self.hv[:, b] = self.hk[:, a], self.hv[:, a]
        self.gto.gto_pages_compact(self.ctx, self.dev, self.k, self.v, t, r, n)
        self.compare()
        assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(r.cpu().numpy(), counts) and n.item() == used
        if take:
            self.host.update(page_table=table, ref_count=counts)
            self.put()

    def write(self, lens):
        self.host["kv_len"] = np.asarray(lens, np.int32)
        self.put()


@pytest.mark.parametrize("dtype,order,page,dh", [("f32", "entry", 4, 16), ("bf16", "head", 8, 32), ("f16", "page", 16, 64), ("bf16", "gaps", 3, 16),
                                                 ("f32", "gaps", 1, 16)])
def test_random_lives_of_a_pool(gto, dtype, order, page, dh):
    rng = np.random.default_rng(page)
    S, width = 7, 9
    p = Pool(gto, S, width, 40, page=page, dh=dh, dtype=dtype, order=order, layers=3)
    copied = 0
    for step in range(60):
        kind = rng.integers(4)
        if kind == 0:
            p.fork(rng.integers(-1, S, S))
        elif kind < 3:
            copied += len(p.resize(rng.integers(-1, width * page + 1, S)))
            lens = p.host["kv_len"].copy()
            for s in range(S):                       # what a sequence holds alone, it may fill
                j = int(lens[s]) // page
                while j < p.host["held"][s] and p.host["ref_count"][p.host["page_table"][s][j]] == 1:
                    lens[s] = rng.integers(lens[s], (j + 1) * page + 1)
                    if lens[s] < (j + 1) * page:
                        break
                    j += 1
            p.write(lens)
        else:
            p.compact()
        pg.check(p.host, page)
    assert copied > 0 or page == 1


@pytest.mark.parametrize("S,n_pages,width", [(1, 1, 1), (1, 5000, 4000), (1500, 9000, 12), (40, 70001, 300)])
def test_sizes(gto, S, n_pages, width):
    rng = np.random.default_rng(S)
    p = Pool(gto, S, width, n_pages, page=4, layers=1, hkv=1, dtype="bf16")
    p.resize(np.minimum(rng.integers(0, width * 4 + 1, S), 4 * (n_pages // S)))
    p.write(np.minimum(p.host["held"] * 4, rng.integers(0, width * 4 + 1, S)))
    p.fork(np.where(rng.random(S) < 0.4, rng.integers(-1, S, S), np.arange(S)))
    p.resize(np.where(rng.random(S) < 0.5, p.host["kv_len"] + rng.integers(0, 9, S), -1).clip(max=width * 4))
    p.compact()
    pg.check(p.host, 4)
    p.resize(np.zeros(S))
    assert (p.host["ref_count"] == 0).all()


def test_a_pool_that_runs_out(gto):
    p = Pool(gto, 5, 4, 8)
    p.resize([16, -1, -1, -1, -1])
    p.resize([8, 12, 16, 4, 2])       # four are left: 12 entries take three of them, no more is served, and 0 gives two back
    assert p.host["held"].tolist() == [2, 3, 0, 0, 0]
    p.resize([8, 12, 8, 4, 2])        # (what came back is there now)
    assert p.host["held"].tolist() == [2, 3, 2, 1, 0]
    p.write([6, 12, 5, 3, 0])
    p.fork([0, 1, 2, 3, 2])
    p.resize([-1, -1, 6, -1, 6])      # two copies of a shared page, and no page
    assert p.host["held"].tolist() == [2, 3, 2, 1, 2]
    p.resize([0, -1, -1, -1, -1])
    assert len(p.resize([-1, -1, 6, -1, 6])) == 2
    pg.check(p.host, 4)


def test_many_sharers_of_one_page(gto):
    """One prompt forked to all others; each then writes into its last page."""
    S = 300
    p = Pool(gto, S, 6, 1000, layers=4, dtype="bf16", hkv=4, dh=32)
    want = np.full(S, -1)
    want[0] = 11
    p.resize(want)
    p.write(np.r_[11, np.zeros(S - 1)])
    p.fork(np.zeros(S))
    assert p.host["ref_count"][:3].tolist() == [S, S, S]
    assert len(p.resize(np.full(S, 20))) == S
    assert p.host["ref_count"][:3].tolist() == [S, S, 0]
    p.fork(np.roll(np.arange(S), 1))      # all change places
    p.fork(np.full(S, -1))
    assert (p.host["ref_count"] == 0).all()


def test_bad_numbers_are_reported_and_left_alone(gto):
    p = Pool(gto, 6, 5, 30)
    p.resize([20, 12, 7, 16, 3, 9])
    p.write([20, 9, 7, 13, 3, 9])
    good = pg.copy_of(p.host)

    def broken(at):
        p.host = pg.copy_of(good)
        for name, where, value in at:
            p.host[name][where] = value
        p.put()

    for at in ([("held", 1, -1)], [("held", 1, 6)], [("kv_len", 1, 13)], [("kv_len", 1, -4)], [("page_table", (1, 0), 30)],
               [("page_table", (1, 2), -1)], [("held", 1, 2 ** 31 - 1)], [("kv_len", 1, 2 ** 31 - 1)]):
        broken(at=at)
        p.fork([1, 1, 2, 2, 4, 5])        # 0 from 1, and 3 from 2, which is sound
        broken(at=at)
        p.fork([0, 2, 1, 3, -1, 5])
        broken(at=at)
        p.resize([-1, 14, -1, 16, -1, 0])
        broken(at=at)
        p.resize([-1, 1, -1, 16, 20, -1])
    broken(at=[])
    p.fork([-2, 6, 2, 2 ** 31 - 1, -2 ** 31, 0])
    broken(at=[])
    p.resize([21, 2 ** 31 - 1, -5, -2 ** 31, 20, 0])


def test_graphs_and_streams(gto):
    p = Pool(gto, 8, 6, 60, layers=2, dtype="bf16")
    p.resize([17, -1, -1, -1, 9, -1, -1, -1])
    p.write([15, 0, 0, 0, 7, 0, 0, 0])
    parent = torch.tensor([0, 0, 0, 0, 4, 4, 4, 4], dtype=torch.int32, device=DEV)
    want = torch.tensor([-1, 18, 19, 20, -1, 8, 9, 10], dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        gto.gto_pages_fork(p.ctx, p.dev, parent)
        gto.gto_pages_resize(p.ctx, p.dev, want, p.k, p.v)
    for turn in range(3):                 # equal each time: the continuations are made anew
        graph.replay()
        torch.cuda.synchronize()
        p.host, bad = pg.fork(p.host, parent.cpu().numpy(), p.page)
        p.host, copies, bad, short = pg.resize(p.host, want.cpu().numpy(), p.page)
        for a, b, n in copies:
            for x in (p.hk, p.hv):
                x[:, b, :n] = x[:, a, :n]
        p.compare()
    want[1:4] = torch.tensor([3, 0, 24])  # other contents
    graph.replay()
    torch.cuda.synchronize()
    p.host, bad = pg.fork(p.host, parent.cpu().numpy(), p.page)
    p.host, copies, bad, short = pg.resize(p.host, want.cpu().numpy(), p.page)
    for a, b, n in copies:
        for x in (p.hk, p.hv):
            x[:, b, :n] = x[:, a, :n]
    p.compare()
    del graph
    torch.cuda.synchronize()
    p.fork([0, 1, 2, 3, 0, 1, 2, 3], stream=side)


def test_caches_beyond_32_bits(gto):
    """9 GB of keys and as many of values in two layers; the pages in use lie at its end."""
    n, page, hkv, dh = 18000, 64, 8, 128
    cfg = gto.make_decode_config(S=2, T=2, n_q_heads=hkv, n_kv_heads=hkv, head_dim=dh, page_size=page, n_pages=n, max_pages=8,
                                 flags=gto.GTO_DECODE_PAGES)
    ctx = gto.gto_decode_create(cfg, 0)
    k, v = (torch.zeros((2, n, page, hkv, dh), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    pool = gto.alloc_page_pool(cfg, DEV)
    pool["page_table"][0, :2] = torch.tensor([n - 1, n - 2], dtype=torch.int32)
    pool["held"][0], pool["kv_len"][0] = 2, 100
    pool["ref_count"][n - 2:] = 1
    for x, a in ((k, 1), (v, 2)):
        x[:, n - 2:].normal_(generator=torch.Generator(DEV).manual_seed(a))
    i32 = dict(dtype=torch.int32, device=DEV)
    gto.gto_pages_fork(ctx, pool, torch.tensor([0, 0], **i32))
    pool["ref_count"][:n - 3] = 1         # so that the only free page is the one before them
    gto.gto_pages_resize(ctx, pool, torch.tensor([-1, 101], **i32), k, v)
    assert gto.gto_decode_status(ctx) == 0 and pool["page_table"][1, :3].tolist() == [n - 1, n - 3, -1]
    for x in (k, v):
        assert torch.equal(x[:, n - 3, :36], x[:, n - 2, :36]) and not x[:, n - 3, 36:].any()
    pool["ref_count"][:n - 3] = 0
    t, r, m = torch.zeros_like(pool["page_table"]), torch.zeros_like(pool["ref_count"]), torch.zeros(1, **i32)
    gto.gto_pages_compact(ctx, pool, k, v, t, r, m)
    assert m.item() == 3 and t[0, :2].tolist() == [2, 1] and t[1, :2].tolist() == [2, 0] and r[:4].tolist() == [1, 1, 2, 0]
    for x in (k, v):
        assert torch.equal(x[:, :3], x[:, n - 3:])
    assert gto.gto_decode_status(ctx) == 0
