"""Decode over shared prefixes of many columns (those that go through shared memory) against the plain 64-bit attention, with inputs in which
what could go wrong decides results: weights that cancel, and keys at the borders that each carry a column's result.

Tolerances: a rounding to a type is off by half a step (finfo.eps / 2 of the value); weights are held in 16 bits and more, cut
off below 2^-15 of themselves; sums and scores as in tests/kv_model.py."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M
from tests.test_attn_shared_plan_cpu import _may
from tests.test_gpu_attn_shared import DEV, INF, NAN, Groups

pytestmark = pytest.mark.gpu

WEIGHTS = 2.0 ** -15


def _half_step(io):
    return torch.finfo(M.DTYPES[io]).eps / 2


@pytest.mark.parametrize("D,page,dtype", [(128, 64, "bf16"), (100, 16, "f16"), (64, 32, "bf16"), (48, 128, "f16"), (256, 64, "bf16"), (132, 32, "f16")])
def test_weights_keep_their_bits(D, page, dtype):
    """Two neighbouring keys of nearly equal weight and opposite values: what is left is small, and an error of a weight shows in it
    whole.  All other keys have weights below e^-40, 16000 of them together below 2^-43: they are not in the sums."""
    print("case: wide weights", D, page, dtype, flush=True)
    prefix, members, H = 16000, 9, 256
    g = Groups([(members, prefix)], [prefix + 3 * s for s in range(members)], 1, D, page, dtype, seed=D)
    b = g.b
    first, second = 4000, 4010
    gen = torch.Generator().manual_seed(D)
    value = torch.randn(D, generator=gen).to(b.dtype)
    for k in b.k:
        k.zero_()
        k[:, 0, 0] = -40.0
    b.k[0][first, 0, 0] = b.k[0][second, 0, 0] = 0.0
    b.k[0][second, 0, 1] = -1.0
    b.v[0][first, 0], b.v[0][second, 0] = value, -value
    g.write()
    q = torch.zeros(members, H, D)
    q[:, :, 0] = 1.0
    q[:, :, 1] = 0.005 + 0.06 * torch.rand(members, H, generator=gen)
    q = q.to(b.dtype)
    out = g.run(H, q.view(members, H * D).to(DEV), 1.0).cpu().view(members, H, D)
    want, tol = M.attention(q, b.k[0][[first, second]], b.v[0][[first, second]], torch.ones(members, 2, dtype=torch.bool), 1.0, _half_step(dtype), WEIGHTS)
    M.check(out, want, tol, "two keys")


def _goes_wide(g_columns, keys, kv_heads, dim, dtype, io):
    return _may(g_columns, keys, kv_heads, dim, io == "f32", io == "f32" and dtype == "bf16")


class Keyed:
    """Groups [(members, prefix, tails), ...] on the device whose keys are random signs, so that a query equal to a key is that key's: it
    has nearly all of the weight, and whatever goes wrong with it shows in its column.  The prefix stands in the first member's pages
    only; what belongs to no token is NaN.  same: the own keys of all sequences are those of the first."""

    def __init__(self, groups, heads, dim, page, dtype, seed, same=False):
        self.heads, self.dim, self.page, self.dtype = heads, dim, page, dtype
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.start, self.prefix, self.lead, self.lens = [0], [], [], []
        for members, prefix, tails in groups:
            self.lead += [len(self.lens)] * members
            self.lens += [prefix + t for t in tails]
            self.prefix.append(prefix)
            self.start.append(len(self.lens))
        self.of = [p for (m, _, _), p in zip(groups, self.prefix) for _ in range(m)]
        width = max(-(-n // page) for n in [*self.lens, *self.prefix]) + 1
        rows, count = [], 0
        for s, n in enumerate(self.lens):
            first = self.of[s] // page if s != self.lead[s] else 0
            last = -(-max(n, self.of[s] if s == self.lead[s] else 0) // page)
            if same and s:
                rows.append(rows[0])
                continue
            rows.append([-1] * first + list(range(count, count + max(0, last - first))) + [-1] * (width - max(first, last)))
            count += max(0, last - first)
        ids = torch.randperm(count + 2, generator=self.gen, device=DEV)
        table = torch.tensor(rows, device=DEV)
        self.table = torch.where(table >= 0, ids[table.clamp(min=0)], -1).to(torch.int32)
        dt, chunks = M.DTYPES[dtype], -(-dim // 8)
        self.k_cache = torch.full((count + 2, heads, chunks, page, 8), NAN, dtype=dt, device=DEV)
        self.v_cache = torch.full((count + 2, heads, page // 8, dim, 8), NAN, dtype=dt, device=DEV)
        self.k, self.v = {}, {}                           # (sequence, whether of the prefix): its tokens
        for s, n in enumerate(self.lens):
            if s == self.lead[s] and self.of[s]:
                self._fill(s, 0, self.of[s], "prefix")
            if n > self.of[s] and not (same and s):
                self._fill(s, self.of[s], n, "own")
            elif same:
                self.k[s, "own"], self.v[s, "own"] = self.k[0, "own"], self.v[0, "own"]

    def _fill(self, s, a, b, which):
        h, d, chunks = self.heads, self.dim, self.k_cache.shape[2]
        dt = self.k_cache.dtype
        k = torch.randint(0, 2, (b - a, h, d), generator=self.gen, device=DEV).mul_(2).sub_(1).to(dt)
        v = torch.randn(b - a, h, d, generator=self.gen, device=DEV).to(dt)
        self.k[s, which], self.v[s, which] = k, v
        pos = torch.arange(a, b, device=DEV)
        page, slot = self.table[s][pos // self.page].long(), pos % self.page
        pad = torch.zeros(b - a, h, 8 * chunks - d, dtype=dt, device=DEV)
        self.k_cache[page, :, :, slot] = torch.cat([k, pad], 2).view(b - a, h, chunks, 8)
        self.v_cache[page, :, slot // 8, :, slot % 8] = v

    def tokens(self, s):
        """Keys and values [len, heads, dim] of sequence s."""
        n, p, empty = self.lens[s], self.of[s], torch.empty(0, self.heads, self.dim, dtype=self.k_cache.dtype, device=DEV)
        return [torch.cat([t[self.lead[s], "prefix"][:min(n, p)] if p else empty, t[s, "own"] if n > p else empty]) for t in (self.k, self.v)]

    def run(self, H, io, scale, pick, window=0, sinks=0, rows=None):
        """pick(s, columns): the positions whose keys are the queries of sequence s, one for each head of a kv head.  Checked: the
        sequences `rows`, every head."""
        n, per = len(self.lens), H // self.heads
        q = torch.zeros(n, self.heads, per, self.dim, device=DEV)
        wanted = {}
        for s in range(n):
            k, v = self.tokens(s)
            at = torch.as_tensor(pick(s, per), device=DEV).clamp(0, max(0, self.lens[s] - 1))
            if self.lens[s]:
                q[s] = k[at].transpose(0, 1)
            if rows is None or s in rows:
                wanted[s] = k, v
        q = q.to(M.DTYPES[io])
        i32 = dict(dtype=torch.int32, device=DEV)
        out = torch.full((n, H * self.dim), NAN, dtype=q.dtype, device=DEV)
        ws = torch.full((B.bitnet_attn_decode_shared_workspace_bytes(n, H, self.heads, self.dim, self.page, self.table.shape[1], window, sinks),), 0xFF,
                        dtype=torch.uint8, device=DEV)
        B.bitnet_attn_decode_shared(q.view(n, -1), torch.tensor(self.start, **i32), torch.tensor(self.prefix, **i32), self.k_cache, self.v_cache,
                                    self.table, torch.tensor(self.lens, **i32), out, scale, window, sinks, ws)
        torch.cuda.synchronize()
        out = out.view(n, self.heads, per, self.dim).double()
        u = 2.0 ** -22                                    # as in kv_model.attention, whose bound this is, a kv head at a time
        for s, (k, v) in wanted.items():
            L = self.lens[s]
            if L == 0:
                assert not out[s].any()
                continue
            j = torch.arange(L, device=DEV)
            seen = (j >= L - window) | (j < sinks) if window else j >= 0
            for h in range(self.heads):
                kh, vh, qh = k[:, h].double()[seen], v[:, h].double()[seen], q[s, h].double()
                x = scale * (qh @ kh.t().contiguous())
                p = torch.softmax(x, 1)
                want, mass = p @ vh, p @ vh.abs()
                score = (self.dim + 16) * u * abs(scale) * qh.abs().sum(1, keepdim=True) + 4 * u * x.abs().amax(1, keepdim=True)    # keys are 1 or -1
                tol = (2 * score + (L + 64) * u + (WEIGHTS if io != "f32" else 0.0)) * mass + _half_step(io) * want.abs() + 1e-30
                off = (out[s, h] - want).abs() / tol
                assert bool((off <= 1.0).all()), f"sequence {s} of {L}, kv head {h}: {float(off.max())} of the tolerance, head {int(off.amax(1).argmax())}"


def _borders(length, prefix, window, sinks):
    """Positions where tiles, quarters of tiles, pages, the prefix, the window or the sinks begin and end, the ends first."""
    low = max(0, length - window) if window else 0
    at = [0, 1, length - 1, length - 2, prefix - 1, prefix, prefix - 2, low, low + 1, low - 1, sinks - 1, sinks]
    for t in range(0, length, 64):
        at += [t, t + 63, t + 15, t + 16, t + 31, t + 32, t + 47, t + 48]
    return [x for x in at if 0 <= x < length]


# heads of 65 to 128 in the cache's type have passes of 256 columns and eight waves, all others of 128 and four
KEYED = [([(9, 8000), (3, 700)], 256, 1, 128, 64, "bf16", "bf16", 0.25), ([(7, 12003), (1, 0)], 160, 1, 100, 16, "f16", "f16", 0.3),
         ([(8, 6016), (7, 5601), (2, 90)], 256, 4, 128, 32, "bf16", "bf16", 0.25), ([(16, 5003), (18, 4500)], 128, 4, 112, 128, "f16", "f16", 0.25),
         ([(96, 2100), (64, 3001)], 32, 8, 64, 16, "bf16", "bf16", 0.35), ([(16, 7000), (20, 6000)], 256, 4, 128, 64, "bf16", "f32", 0.25),
         ([(24, 5003), (32, 4100)], 128, 4, 80, 32, "f16", "f32", 0.3), ([(12, 5003), (10, 4500)], 256, 4, 256, 64, "bf16", "bf16", 0.15),
         ([(24, 9000), (28, 8200)], 256, 4, 256, 16, "bf16", "f32", 0.15), ([(20, 8000), (16, 9000)], 256, 4, 256, 256, "f16", "f32", 0.15),
         ([(32, 9000), (1, 100), (1, 300)], 40, 10, 64, 32, "f16", "f32", 0.35)]


@pytest.mark.parametrize("window,sinks", [(0, 0), (3500, 130)])
@pytest.mark.parametrize("groups,H,Hkv,D,page,dtype,io,scale", KEYED)
def test_every_key_counts(groups, H, Hkv, D, page, dtype, io, scale, window, sinks):
    """Several kv heads, several passes, two wide groups in one line, narrow ones beside them; the columns of a group go through the
    borders of all tiles.  A member as long as the prefix, one that is shorter, others longer."""
    print("case: keyed", groups, H, Hkv, D, page, dtype, io, window, flush=True)
    tails = lambda m: ([300, 0, -77] + [1 + 13 * i for i in range(m)])[:m]  # noqa: E731
    g = Keyed([(m, p, tails(m) if p > 100 else [40 + i for i in range(m)]) for m, p in groups], Hkv, D, page, dtype, seed=D + H)
    for m, p in groups:
        if p > 2000:
            assert _goes_wide(m * H // Hkv, p, Hkv, D, dtype, io), "the case has to go through shared memory"

    def pick(s, per):
        at = _borders(g.lens[s], g.of[s], window, sinks)
        first = (s - g.lead[s]) * per
        return [at[(c if c < 12 else 12 + first + c - 12) % len(at)] for c in range(per)]
    g.run(H, io, scale, pick, window, sinks)


@pytest.mark.parametrize("dtype,io,D,page", [("bf16", "bf16", 128, 32), ("f16", "f16", 100, 16), ("bf16", "f32", 128, 64), ("f16", "f32", 100, 128), ("bf16", "bf16", 256, 64)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (8500, 300)])
def test_missing_pages_and_values_that_are_not_finite(dtype, io, D, page, window, sinks):
    print("case: wide missing, infinite", dtype, io, D, page, window, flush=True)
    prefix, members, H = 9001, 16, 256
    assert _goes_wide(members * H, prefix, 1, D, dtype, io)
    g = Groups([(members, prefix)], [prefix + t for t in (0, 3, 64, 500, 1, 2, -9, 4, *range(8))], 1, D, page, dtype, seed=D)
    b = g.b
    table = b.table.clone()
    for at, x in ((2000, -1), (7000, 10 ** 7), (8990, -2 ** 31)):
        b.table[0, at // page] = x
    check = lambda scale, rows: _checked(g, H, io, scale, window, sinks, rows)  # noqa: E731
    check(1 / math.sqrt(D), [0, 3, 6, 15])
    b.table.copy_(table)
    for s, at, ch, x in ((0, 3, 1, INF), (0, 5000, 2, -INF), (0, 8999, 0, NAN), (0, 100, 5, INF), (0, 7000, 5, -INF), (0, 9000, D - 1, INF),
                         (1, prefix + 1, 3, INF), (3, prefix + 150, 2, INF), (3, prefix + 151, D - 2, -INF)):
        b.v[s][at, 0, ch] = x
    g.write()
    check(0.1, [0, 1, 3, 6, 15])


def _checked(g, H, io, scale, window, sinks, rows):
    """Groups.run against kv_model.attention, with weights held as everywhere."""
    b = g.b
    q = torch.randn(len(b.lens), H * b.dim, generator=torch.Generator().manual_seed(1)).to(M.DTYPES[io])
    out = g.run(H, q.to(DEV), scale, window, sinks).cpu().view(-1, H, b.dim)
    for s in rows:
        n = b.lens[s]
        seen = M.visible(torch.tensor([n - 1]), n, window, sinks) & g.there(s)[None]
        want, tol = M.attention(q[s].view(1, H, b.dim), b.k[s], b.v[s], seen, scale, _half_step(io), WEIGHTS if io != "f32" else 0.0)
        M.check(out[s][None], want, tol, f"sequence {s} of {n}")


# Shares of more than 64 tiles, whose page numbers are asked for again in between (256 work groups).
@pytest.mark.parametrize("window,sinks", [(0, 0), (25000, 30000)])
@pytest.mark.parametrize("members,H,Hkv,D,page,dtype,io,scale,prefix", [(12, 256, 2, 128, 16, "bf16", "f32", 0.25, 65536), (20, 256, 4, 128, 64, "bf16", "bf16", 0.25, 61000),
                                                                      (20, 512, 4, 64, 32, "f16", "f16", 0.35, 65536), (12, 256, 2, 256, 128, "bf16", "bf16", 0.15, 65000)])
def test_shares_of_many_tiles(members, H, Hkv, D, page, dtype, io, scale, prefix, window, sinks):
    print("case: wide refills", members, H, Hkv, D, page, dtype, io, window, flush=True)
    width = 256 if io != "f32" and 64 < D <= 128 else 128
    tiles = -(-prefix // 64) if not window else (sinks + window) // 64
    groups = 512 if D <= 64 else 256
    assert _goes_wide(members * H // Hkv, prefix, Hkv, D, dtype, io)
    assert Hkv * -(-members * H // Hkv // width) * tiles // groups >= 64
    g = Keyed([(members, prefix, [200 + 3 * i for i in range(members)])], Hkv, D, page, dtype, seed=D)
    step = -(-tiles // (members * (H // Hkv)))            # the columns of all members go through all tiles that are seen

    def pick(s, per):
        t = (torch.arange(per) + s * per) * max(1, step) % tiles
        at = t * 64 + (t * 37 + s) % 64
        return torch.where(at < sinks, at, at - sinks + g.lens[s] - window) if window else at
    g.run(H, io, scale, pick, window, sinks)


# Shares of more than 512 units, whose page numbers go through shared memory in turns: own rows of 64 sequences over the same pages.
@pytest.mark.parametrize("window,sinks", [(0, 0), (14000, 18000)])
@pytest.mark.parametrize("H,D,page,dtype,io,scale", [(128, 64, 16, "bf16", "f32", 0.35), (128, 64, 32, "f16", "f16", 0.35), (64, 128, 256, "bf16", "bf16", 0.25)])
def test_shares_of_many_units(H, D, page, dtype, io, scale, window, sinks):
    print("case: narrow refills", H, D, page, dtype, io, window, flush=True)
    length, Hkv, n = 33000, 8, 64
    assert n * Hkv * (length if not window else window + sinks) // 32 // 512 > 900
    g = Keyed([(1, 0, [length])] * n, Hkv, D, page, dtype, seed=D, same=True)

    def pick(s, per):
        at = (torch.arange(per) * 2053 + s * 32 * 17 + s % 32) % (length if not window else sinks + window)
        at[0] = 512 * 32 + 7                              # around the 512th unit of a row
        at[1] = 512 * 32 - 5
        return torch.where(at < sinks, at, at - sinks + length - window) if window else at
    g.run(H, io, scale, pick, window, sinks, rows=range(0, n, 3))


@pytest.mark.parametrize("D,dtype,io", [(128, "bf16", "bf16"), (100, "f16", "f32"), (64, "bf16", "f32"), (256, "bf16", "bf16")])
def test_the_same_bits_in_every_replay_and_on_another_stream(D, dtype, io):
    """A wide call captured into a graph and replayed over other contents, with eager calls and other work on its workspace between."""
    print("case: wide graph", D, dtype, io, flush=True)
    H, Hkv, members, prefix = 128, 2, 24, 9000
    assert _goes_wide(members * H // Hkv, prefix, Hkv, D, dtype, io)
    g = Keyed([(members, prefix, [50 + i for i in range(members)]), (3, 40, [5, 60, 7])], Hkv, D, 64, dtype, seed=D)
    n, i32 = members + 3, dict(dtype=torch.int32, device=DEV)
    first = torch.randn(n, H * D, generator=g.gen, device=DEV).to(M.DTYPES[io])
    second = torch.randn(n, H * D, generator=g.gen, device=DEV).to(M.DTYPES[io])
    start, prefixes, lens = torch.tensor(g.start, **i32), torch.tensor(g.prefix, **i32), torch.tensor(g.lens, **i32)
    need = B.bitnet_attn_decode_shared_workspace_bytes(n, H, Hkv, D, 64, g.table.shape[1])
    q, out, ws = first.clone(), torch.empty_like(first), torch.empty(need, dtype=torch.uint8, device=DEV)
    call = lambda q, out, ws: B.bitnet_attn_decode_shared(q, start, prefixes, g.k_cache, g.v_cache, g.table, lens, out, 0.08, ws=ws)  # noqa: E731
    want = {}
    for name, x in (("first", first), ("second", second)):
        want[name] = torch.empty_like(x)
        call(x, want[name], torch.full_like(ws, 0xFF))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(q, out, ws)
        assert torch.equal(out, want["first"])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call(q, out, ws)
    torch.cuda.synchronize()
    for turn in range(4):
        name, x = (("second", second), ("first", first))[turn % 2]
        q.copy_(x)
        ws.fill_(0x7F + turn)
        out.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[name]), turn
        again = torch.empty_like(out)
        call(x, again, torch.empty_like(ws))
        assert torch.equal(again, want[name]), turn
