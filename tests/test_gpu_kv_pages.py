"""GPU parity of the cache's bookkeeping: tokens written into their pages, and pages reserved, forked, freed, trimmed, copied
and compacted, against plain models; every value bit for bit.  The last tests run the calls together, also in a HIP graph."""
import random

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _announce(*what):
    print("case:", *what, flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _bits(t):
    return t.cpu().view(torch.int16)


# ---------------------------------------------------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("src", ["f32", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,D,page", [(8, 128, 16), (3, 100, 64), (2, 4, 32), (1, 256, 256), (5, 36, 128)])
def test_append(H, D, page, dtype, src):
    _announce("append", H, D, page, dtype, src)
    new = [1, 0, 2, 7, 8, 9, 40, 300, 5]
    past = [0, 9, 15, 3, 8, 100, 1, 0, 251]
    lens = [n + p for n, p in zip(new, past)]
    b = M.Batch(lens, H, D, page, dtype, seed=H + D, fill=3.0)
    before = b.on(DEV)
    g = torch.Generator().manual_seed(5)
    k = torch.randn(sum(new), H, D, generator=g) * 3
    v = torch.randn(sum(new), H, D, generator=g) * 3
    k[0, 0, 0], v[-1, -1, -1] = float("inf"), float("nan")
    if src == "cache":
        k, v = k.to(b.dtype), v.to(b.dtype)
    start = [0]
    for s, n in enumerate(new):
        if n:
            b.write(s, lens[s] - n, k[start[-1]:start[-1] + n].to(b.dtype), v[start[-1]:start[-1] + n].to(b.dtype))
        start.append(start[-1] + n)
    kc, vc, table, kv_len = before
    B.bitnet_kv_append(k.to(DEV), v.to(DEV), _i32(start), kc, vc, table, kv_len)
    torch.cuda.synchronize()
    keep = torch.isnan(b.v_cache)
    assert torch.equal(_bits(kc), _bits(b.k_cache))
    assert torch.equal(torch.isnan(vc.cpu()), keep) and torch.equal(_bits(vc)[~keep], _bits(b.v_cache)[~keep])


@pytest.mark.parametrize("given", [True, False])
def test_append_one_token_each(given):
    _announce("append one each", given)
    lens = [1, 16, 17, 40, 0, 33]
    b = M.Batch(lens, 4, 64, 16, "bf16", seed=1, fill=0.5)
    kc, vc, table, kv_len = b.on(DEV)
    k, v = torch.randn(6, 4, 64), torch.randn(6, 4, 64)
    for s, n in enumerate(lens):
        if n:                                  # a length of 0 has no place for its token
            b.write(s, n - 1, k[s:s + 1].to(b.dtype), v[s:s + 1].to(b.dtype))
    B.bitnet_kv_append(k.view(6, -1).to(DEV), v.view(6, -1).to(DEV), _i32(list(range(7))) if given else None, kc, vc, table, kv_len)
    torch.cuda.synchronize()
    assert torch.equal(_bits(kc), _bits(b.k_cache)) and torch.equal(_bits(vc), _bits(b.v_cache))


def test_append_leaves_out_what_has_no_place():
    _announce("append without places")
    b = M.Batch([20, 50, 40], 2, 64, 16, "bf16", seed=2, fill=0.5)
    b.table[1, 1] = -1
    b.table[2, 0] = b.pages                    # past the pool
    kc, vc, table, kv_len = b.on(DEV)
    kv_len[0] = 10                             # 30 new tokens of which 20 lie below position 0
    kv_len[2] = 10 ** 8                        # past the row of the table
    k = torch.randn(30 + 50 + 3, 2, 64)
    for p in range(10):
        b.write(0, p, k[20 + p:21 + p].to(b.dtype), k[20 + p:21 + p].to(b.dtype))
    for p in list(range(16)) + list(range(32, 50)):
        b.write(1, p, k[30 + p:31 + p].to(b.dtype), k[30 + p:31 + p].to(b.dtype))
    B.bitnet_kv_append(k.to(DEV), k.to(DEV), _i32([0, 30, 80, 83]), kc, vc, table, kv_len)
    torch.cuda.synchronize()
    assert torch.equal(_bits(kc), _bits(b.k_cache)) and torch.equal(_bits(vc), _bits(b.v_cache))


# ---------------------------------------------------------------------------------------------------------------------
# Pages
# ---------------------------------------------------------------------------------------------------------------------
class Device:
    """The same state on the GPU, with pages whose contents name them."""

    def __init__(self, m, layers=2, heads=1, dim=12):
        self.m = m
        page, pages = m.page, m.n_pages
        self.k = torch.zeros(layers, pages, heads, -(-dim // 8), page, 8, dtype=torch.bfloat16, device=DEV)
        self.v = torch.zeros(layers, pages, heads, page // 8, dim, 8, dtype=torch.bfloat16, device=DEV)
        self.label(self.k)[:] = self.names(pages, layers, 0)
        self.label(self.v)[:] = self.names(pages, layers, 1)
        self.table, self.lens, self.refs = _i32(m.table), _i32(m.lens), _i32(m.refs)
        self.count = _i32([-1])
        self.ws = torch.full((B.bitnet_kv_workspace_bytes(pages, len(m.lens)),), 0xFF, dtype=torch.uint8, device=DEV)

    @staticmethod
    def label(pool):
        return pool.view(torch.int16).view(pool.shape[0], pool.shape[1], -1)

    @staticmethod
    def names(pages, layers, which):
        return ((torch.arange(pages)[None, :] * 7 + 2 * torch.arange(layers)[:, None] + which) % 32000).to(torch.int16).to(DEV)[:, :, None]

    def check(self, holds=True):
        torch.cuda.synchronize()
        m = self.m
        assert self.table.tolist() == m.table and self.lens.tolist() == m.lens and self.refs.tolist() == m.refs
        if holds:
            live = torch.tensor(m.refs) > 0
            for which, pool in ((0, self.k), (1, self.v)):
                want = self.names(m.n_pages, pool.shape[0], which)[:, torch.tensor(m.holds)]
                got = self.label(pool)
                assert torch.equal(got[:, live], want[:, live].expand_as(got[:, live]))


@pytest.mark.parametrize("n_seqs,width,pages,page", [(5, 6, 40, 16), (40, 9, 300, 32), (1100, 4, 5000, 16), (7, 300, 9000, 64)])
def test_reserve(n_seqs, width, pages, page):
    _announce("reserve", n_seqs, width, pages, page)
    r = random.Random(pages)
    m = M.Pages(n_seqs, width, pages, page)
    for p in r.sample(range(pages), pages // 3):          # pages that others hold
        m.refs[p] = r.randint(1, 3)
    d = Device(m)
    for _ in range(4):
        seqs = r.sample(range(n_seqs), r.randint(1, n_seqs))
        n_new = [r.choice([0, 1, 1, page, page - 1, r.randint(0, width * page // 2)]) for _ in seqs]
        short = m.reserve(seqs, n_new)
        B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32(seqs), _i32(n_new), page, d.count, d.ws)
        d.check(holds=False)
        assert d.count.item() == short


def test_reserve_refusals_on_the_device():
    _announce("reserve refusals")
    m = M.Pages(4, 3, 5, 16)
    d = Device(m)
    seqs, n_new = [0, 99, 1, -3, 2, 3], [17, 5, 49, 1, -1, 70000]
    d = Device(M.Pages(6, 3, 5, 16))
    m = d.m
    assert m.reserve(seqs, n_new) == 5
    B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32(seqs), _i32(n_new), 16, d.count, d.ws)
    d.check(holds=False)
    assert d.count.item() == 5
    # 3 pages left: the second does not fit, so later ones find none either, but those that need none are served
    seqs, n_new = [1, 2, 3, 0], [16, 48, 16, 15]
    assert m.reserve(seqs, n_new) == 2
    B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32(seqs), _i32(n_new), 16, d.count, d.ws)
    d.check(holds=False)
    assert d.count.item() == 2


@pytest.mark.parametrize("page,layers,heads,dim", [(16, 2, 1, 12), (32, 3, 2, 100), (128, 1, 4, 128)])
def test_fork_free_trim_compact(page, layers, heads, dim):
    _announce("life of a pool", page, layers, heads, dim)
    r = random.Random(page)
    m = M.Pages(24, 12, 160, page)
    d = Device(m, layers, heads, dim)
    empty = set(range(24))
    for step in range(30):
        used = sorted(set(range(24)) - empty)
        what = r.choice(["new", "grow", "fork", "fork", "free", "trim", "compact"])
        if what in ("new", "grow"):
            pick = sorted(empty) if what == "new" else used
            pick = r.sample(pick, min(len(pick), r.randint(1, 5)))
            n_new = [r.randint(1, 3 * page) for _ in pick]
            short = m.reserve(pick, n_new)
            B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32(pick), _i32(n_new), page, d.count, d.ws)
            assert d.count.item() == short
            empty = {s for s in range(24) if m.lens[s] == 0}
        elif what == "fork" and used and empty:
            kids = r.sample(sorted(empty), min(len(empty), r.randint(1, 6)))
            parents = [r.choice(used) for _ in kids]
            short = m.fork(parents, kids)
            B.bitnet_kv_fork(d.k, d.v, d.table, d.lens, d.refs, _i32(parents), _i32(kids), d.count, d.ws)
            assert d.count.item() == short
            empty -= {k for k in kids if m.lens[k]}
        elif what == "free" and used:
            gone = r.sample(used, r.randint(1, min(4, len(used))))
            m.free(gone)
            B.bitnet_kv_free(d.table, d.lens, d.refs, _i32(gone + gone[:1] + [-1]))      # twice and out of range: once
            empty |= set(gone)
        elif what == "trim" and used:
            window, sinks = r.choice([1, page, 2 * page + 3]), r.choice([0, 4, page + 1])
            m.trim(used, window, sinks)
            B.bitnet_kv_trim(d.table, d.lens, d.refs, _i32(used), page, window, sinks)
        elif what == "compact":
            live = m.compact()
            B.bitnet_kv_compact(d.k, d.v, d.table, d.refs, d.count, d.ws)
            assert d.count.item() == live
        d.check()


def test_fork_when_pages_run_out():
    _announce("fork out of pages")
    m = M.Pages(6, 4, 5, 16)
    assert m.reserve([0, 1], [20, 16]) == 0               # 3 pages taken, 2 left
    d = Device(m)
    parents, kids = [0, 1, 0, 0, 9, 5], [2, 3, 4, 5, 1, 5]
    short = m.fork(parents[:4], kids[:4]) + 2
    B.bitnet_kv_fork(d.k, d.v, d.table, d.lens, d.refs, _i32(parents), _i32(kids), d.count, d.ws)
    d.check()
    assert d.count.item() == short == 3 and m.lens[5] == 0 and m.lens[3] == 16


@pytest.mark.parametrize("pages,live", [(1, 0), (1, 1), (64, 0), (64, 64), (100, 1), (2047, 1000), (2048, 2000), (2049, 30), (9001, 4500)])
def test_compact_sizes(pages, live):
    _announce("compact", pages, live)
    r = random.Random(pages + live)
    m = M.Pages(3, 3001, pages, 16)
    ids = r.sample(range(pages), live)
    for i, p in enumerate(ids):
        m.table[i % 3][i // 3] = p
        m.refs[p] = 1 + i % 2
    d = Device(m, layers=1)
    assert m.compact() == live
    B.bitnet_kv_compact(d.k, d.v, d.table, d.refs, d.count, d.ws)
    d.check()
    assert d.count.item() == live


def test_copy_pages():
    _announce("copy pages")
    m = M.Pages(1, 1, 50, 64)
    m.refs = [1] * 50
    d = Device(m, layers=3, heads=3, dim=100)
    src, dst = [0, 7, 49, 3, -1, 50], [10, 11, 12, -1, 13, 14]
    for s, t in list(zip(src, dst))[:3]:
        m.holds[t] = s
    B.bitnet_kv_copy_pages(d.k, d.v, _i32(src), _i32(dst))
    d.check()


def test_empty_calls():
    _announce("empty calls")
    m = M.Pages(3, 2, 8, 16)
    d = Device(m)
    none = _i32([])
    B.bitnet_kv_free(d.table, d.lens, d.refs, none)
    B.bitnet_kv_trim(d.table, d.lens, d.refs, none, 16, 4)
    B.bitnet_kv_reserve(d.table, d.lens, d.refs, none, none, 16, d.count, d.ws)
    assert d.count.item() == 0
    d.count.fill_(-1)
    B.bitnet_kv_fork(d.k, d.v, d.table, d.lens, d.refs, none, none, d.count, d.ws)
    assert d.count.item() == 0
    B.bitnet_kv_copy_pages(d.k, d.v, none, none)
    k, v = d.k[0], d.v[0]
    empty = torch.empty(0, 12, device=DEV)
    B.bitnet_kv_append(empty, empty, _i32([0, 0, 0, 0]), k, v, d.table, d.lens)
    B.bitnet_attn_prefill(empty, _i32([0, 0, 0, 0]), k, v, d.table, d.lens, empty.clone(), 1.0)
    B.bitnet_attn_decode(empty, k, v, d.table[:0], d.lens[:0], empty.clone(), 1.0)
    d.check()


# ---------------------------------------------------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------------------------------------------------
def test_window_with_pages_given_back():
    """What trim gives back is never seen again: attention before and after it is the same, bit for bit."""
    _announce("trim and attend")
    b = M.Batch([700, 90, 33], 2, 64, 16, "bf16", seed=3)
    k, v, table, lens = b.on(DEV)
    refs = torch.zeros(b.pages, dtype=torch.int32, device=DEV)
    refs[table[table >= 0].long()] = 1
    q = torch.randn(3, 4 * 64, device=DEV)
    ws = torch.empty(max(16, B.bitnet_attn_decode_workspace_bytes(3, 4, 2, 64, 16, table.shape[1], 50, 5)), dtype=torch.uint8, device=DEV)
    first, second = torch.empty_like(q), torch.empty_like(q)
    B.bitnet_attn_decode(q, k, v, table, lens, first, 0.125, 50, 5, ws)
    lens -= 1                                  # as the step before: its trim leaves what this step sees
    B.bitnet_kv_trim(table, lens, refs, _i32([0, 1, 2]), 16, 50, 5)
    lens += 1
    gone = refs == 0
    assert int(gone.sum()) > 2 + 35            # two spares, and most of the first sequence
    k[gone], v[gone] = float("nan"), float("nan")
    B.bitnet_attn_decode(q, k, v, table, lens, second, 0.125, 50, 5, ws)
    torch.cuda.synchronize()
    assert torch.equal(first, second)


def test_decode_step_in_a_graph():
    """reserve, append, decode captured once: every replay is the next token, equal to the same step made eagerly."""
    _announce("decode step in a graph")
    n, H, Hkv, D, page, width, pages = 3, 8, 2, 128, 16, 40, 130

    def state():
        m = M.Pages(n, width, pages, page)
        d = Device(m, 1, Hkv, D)
        B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32([0, 1, 2]), _i32([14, 300, 1]), page, d.count, d.ws)
        g = torch.Generator(device=DEV).manual_seed(4)
        d.k.copy_(torch.randn(d.k.shape, device=DEV, generator=g))
        d.v.copy_(torch.randn(d.v.shape, device=DEV, generator=g))
        d.x = torch.zeros(n, (H + 2 * Hkv) * D, device=DEV)
        d.q, d.kk, d.vv = (torch.zeros(n, w * D, device=DEV) for w in (H, Hkv, Hkv))
        d.out = torch.empty(n, H * D, device=DEV)
        d.seqs, d.one = _i32([0, 1, 2]), _i32([1, 1, 1])
        d.aws = torch.empty(B.bitnet_attn_decode_workspace_bytes(n, H, Hkv, D, page, width), dtype=torch.uint8, device=DEV)
        return d

    def step(d, stream):
        B.bitnet_kv_reserve(d.table, d.lens, d.refs, d.seqs, d.one, page, d.count, d.ws, stream)
        B.bitnet_kv_append(d.kk, d.vv, None, d.k[0], d.v[0], d.table, d.lens, stream)
        B.bitnet_attn_decode(d.q, d.k[0], d.v[0], d.table, d.lens, d.out, 0.09, 0, 0, d.aws, stream)

    def fill(d, i):
        g = torch.Generator(device=DEV).manual_seed(100 + i)
        for t in (d.q, d.kk, d.vv):
            t.normal_(generator=g)

    eager, captured = state(), state()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    saved = [t.clone() for t in (captured.table, captured.lens, captured.refs)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(captured, side)
    torch.cuda.synchronize()
    for t, s in zip((captured.table, captured.lens, captured.refs), saved):
        assert torch.equal(t, s), "capturing runs nothing"
    for i in range(5):
        fill(eager, i)
        step(eager, None)
        fill(captured, i)
        torch.cuda.synchronize()
        captured.out.fill_(float("nan"))
        captured.aws.fill_(0xFF)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        assert captured.count.item() == 0 and captured.lens.tolist() == [15 + i, 301 + i, 2 + i]
        for t in ("out", "table", "lens", "refs", "k", "v"):
            assert torch.equal(getattr(eager, t), getattr(captured, t)), (i, t)


def test_reserve_keeps_the_order_of_its_list():
    _announce("reserve in order")
    for want, short in (([10, 1, 0], 2), ([1, 10, 1], 2), ([1, 1, 10], 1), ([2, 3, 0], 0)):
        d = Device(M.Pages(3, 12, 5, 16))
        n_new = [16 * w for w in want]
        assert d.m.reserve([0, 1, 2], n_new) == short
        B.bitnet_kv_reserve(d.table, d.lens, d.refs, _i32([0, 1, 2]), _i32(n_new), 16, d.count, d.ws)
        d.check(holds=False)
        assert d.count.item() == short
