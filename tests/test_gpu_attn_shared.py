"""Decode over shared prefixes against the plain 64-bit attention: groups of one sequence to many, prefixes of nothing to tens of
thousands of tokens that end anywhere in a page, every type, odd heads, windows, missing pages, offsets that are wrong, and
values that are not finite.  Tolerances follow from the arithmetic (tests/kv_model.py)."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


class Groups:
    """Groups [(members, prefix), ...] whose sequences have the given lengths.  Keys and values of the prefix stand in the first
    member's pages only: the others' rows name nothing there, and their last page of it holds NaN below its end."""

    def __init__(self, groups, lens, heads, dim, page, dtype, seed, width=None):
        self.groups, self.b = groups, M.Batch(lens, heads, dim, page, dtype, seed, width=width)
        self.start = [0]
        b = self.b
        for members, prefix in groups:
            first = self.start[-1]
            for s in range(first, first + members):
                if s > first:
                    b.table[s, :prefix // page] = -1
                    n = min(prefix, lens[s])
                    b.k[s][:n], b.v[s][:n] = b.k[first][:n], b.v[first][:n]
                    if n == prefix and lens[s] > prefix and prefix % page:       # the page that the prefix ends in
                        low = prefix // page * page
                        nan = torch.full((prefix - low, heads, dim), NAN, dtype=b.dtype)
                        b.write(s, low, nan, nan)
            self.start.append(first + members)

    def write(self):
        """The sequences' k and v again, after a change: the prefix into the first member's pages, the rest into each one's own."""
        b = self.b
        for g, (members, prefix) in enumerate(self.groups):
            first = self.start[g]
            for s in range(first, first + members):
                n = min(prefix, b.lens[s])
                if s == first:
                    b.write(s, 0, b.k[s], b.v[s])
                else:
                    b.k[s][:n], b.v[s][:n] = b.k[first][:n], b.v[first][:n]
                    if b.lens[s] > n:
                        b.write(s, n, b.k[s][n:], b.v[s][n:])

    def there(self, s):
        """Whether the tokens of sequence s have pages: below the prefix the first member's."""
        b = self.b
        g = max(i for i in range(len(self.groups)) if self.start[i] <= s and self.groups[i][0] > 0)
        first, prefix = self.start[g], self.groups[g][1]
        own, lead = ((b.table[i] >= 0) & (b.table[i] < b.pages) for i in (s, first))
        at = torch.arange(b.lens[s])
        return torch.where(at < prefix, lead[at // b.page], own[at // b.page])

    def arrays(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        return torch.tensor(self.start, **i32), torch.tensor([p for _, p in self.groups], **i32)

    def run(self, H, q, scale, window=0, sinks=0, arrays=None, tensors=None, stream=None, fill=NAN):
        b = self.b
        k, v, table, lens = tensors or b.on(DEV)
        start, prefix = arrays or self.arrays()
        out = torch.full_like(q, fill)
        need = B.bitnet_attn_decode_shared_workspace_bytes(len(b.lens), H, b.heads, b.dim, b.page, table.shape[1], window, sinks)
        ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)     # NaN patterns: nothing in it may matter
        B.bitnet_attn_decode_shared(q, start, prefix, k, v, table, lens, out, scale, window, sinks, ws, stream)
        torch.cuda.synchronize()
        return out

    def check(self, out, H, q, scale, io, window=0, sinks=0, rows=None):
        b = self.b
        out = out.cpu().view(-1, H, b.dim)
        for s in range(len(b.lens)) if rows is None else rows:
            n = b.lens[s]
            if n == 0:
                assert not out[s].any(), "an empty sequence gives zeros"
                continue
            seen = M.visible(torch.tensor([n - 1]), n, window, sinks) & self.there(s)[None]
            # weights of the cache's type keep 2^-15; over the prefix of many columns each is rounded to it once (by half a step h at
            # most) and summed as rounded: h of the weighted sum, and h of the sum that divides it
            members = max((m for m, _ in self.groups), default=0)
            half = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[io]
            weights = 2 * half if members * (H // b.heads) > 64 else 2.0 ** -15 if io != "f32" else 0.0
            want, tol = M.attention(q[s].view(1, H, b.dim), b.k[s], b.v[s], seen, scale, M.io_eps(io), weights)
            M.check(out[s][None], want, tol, f"sequence {s} of {n}")

    def run_and_check(self, H, io, seed, window=0, sinks=0, scale=None, rows=None):
        scale = 1 / math.sqrt(self.b.dim) if scale is None else scale
        q = torch.randn(len(self.b.lens), H * self.b.dim, generator=torch.Generator().manual_seed(seed)).to(M.DTYPES[io])
        self.check(self.run(H, q.to(DEV), scale, window, sinks), H, q, scale, io, window, sinks, rows)


def _announce(*what):
    print("case:", *what, flush=True)


# prefixes that end everywhere in pages and units, tails from nothing on, a group of one, an empty group, one without a prefix
GROUPS = [(3, 37), (1, 64), (0, 5), (4, 0), (2, 1), (5, 160), (1, 0), (9, 333)]
TAILS = [1, 0, 30, 7, 5, 60, 0, 300, 0, 63, 1, 2, 31, 32, 33, 100, 19, 0, 1, 15, 16, 17, 250, 64, 3]
LENS = [p + t for (m, p), ts in zip([g for g in GROUPS if g[0]], [TAILS[:3], TAILS[3:4], TAILS[4:8], TAILS[8:10], TAILS[10:15], TAILS[15:16], TAILS[16:25]])
        for t in ts]
SIZES = [(4, 1, 128, 16), (32, 8, 128, 32), (3, 3, 100, 64), (6, 2, 64, 128), (5, 1, 256, 256), (16, 1, 80, 16), (17, 1, 20, 32),
         (40, 1, 132, 16), (4, 2, 4, 16), (72, 1, 64, 32), (10, 5, 96, 32)]


@pytest.mark.parametrize("io", ["f32", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D,page", SIZES)
def test_groups(H, Hkv, D, page, dtype, io):
    _announce("shared", H, Hkv, D, page, dtype, io)
    Groups(GROUPS, LENS, Hkv, D, page, dtype, seed=H + D).run_and_check(H, dtype if io == "cache" else io, seed=1)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (31, 70), (64, 32), (100, 33), (200, 150), (1000, 5), (150, 10 ** 9), (10 ** 12, 3)])
@pytest.mark.parametrize("H,Hkv,D,page,dtype,io", [(8, 2, 128, 16, "bf16", "f32"), (4, 4, 100, 64, "f16", "f32"), (4, 1, 64, 32, "bf16", "bf16")])
def test_window_and_sinks(H, Hkv, D, page, dtype, io, window, sinks):
    _announce("shared window", H, Hkv, D, page, dtype, io, window, sinks)
    Groups(GROUPS, LENS, Hkv, D, page, dtype, seed=D + 7).run_and_check(H, io, seed=2, window=window, sinks=sinks)


@pytest.mark.parametrize("groups,tail,H,Hkv,D,page,dtype,io", [
    ([(2, 20011)], 100, 4, 1, 64, 16, "bf16", "f32"), ([(64, 1500)], 33, 4, 1, 128, 32, "bf16", "bf16"), ([(20, 900)], 400, 8, 2, 128, 64, "f16", "f16"),
    ([(33, 700), (2, 5000)], 65, 2, 2, 256, 64, "bf16", "bf16"), ([(70, 300)], 1, 32, 1, 36, 32, "f16", "f32"), ([(1, 9000), (3, 2000)], 3000, 8, 8, 128, 128, "bf16", "f32"),
    ([(100, 257)], 5, 1, 1, 100, 16, "f16", "f32"), ([(12, 4099), (7, 2500), (5, 1)], 600, 6, 6, 100, 64, "f16", "f32")])
def test_many_and_long(groups, tail, H, Hkv, D, page, dtype, io):
    _announce("shared long", groups, H, Hkv, D, page, dtype, io)
    lens = [p + (17 * i + 5) % (tail + 1) for m, p in groups for i in range(m)]
    n = len(lens)
    rows = None if n < 12 else sorted({0, 1, n // 3, n // 2, n - 2, n - 1})
    Groups(groups, lens, Hkv, D, page, dtype, seed=3).run_and_check(H, io, seed=3, rows=rows)


# Prefixes that go through shared memory: many columns (members times heads of a kv head) behind enough keys.
WIDE = [(4, 256, 1, 64, 16, "bf16", "bf16", 6000), (6, 200, 1, 48, 64, "f16", "f16", 5003), (9, 256, 1, 64, 32, "bf16", "f32", 8011),
        (5, 256, 1, 128, 32, "bf16", "bf16", 9001), (7, 150, 1, 100, 16, "f16", "f16", 12000), (16, 256, 1, 128, 64, "bf16", "f32", 9000),
        (16, 256, 1, 100, 16, "f16", "f32", 6100), (5, 256, 1, 256, 128, "bf16", "bf16", 6007), (12, 256, 1, 132, 32, "f16", "f32", 9000)]


@pytest.mark.parametrize("members,H,Hkv,D,page,dtype,io,prefix", WIDE)
def test_wide_prefixes(members, H, Hkv, D, page, dtype, io, prefix):
    """Beside a group of one sequence and a small one; a member as long as the prefix, one that is shorter, one longer."""
    _announce("shared wide", members, H, D, page, dtype, io, prefix)
    tails = [37, 0, -100, 300] + [5] * (members - 4)
    lens = [40] + [prefix + t for t in tails] + [70, 90, 64]
    Groups([(1, 0), (members, prefix), (3, 64)], lens, Hkv, D, page, dtype, seed=14).run_and_check(H, io, seed=14, rows=[0, 1, 2, 3, 4, members, members + 3])


@pytest.mark.parametrize("window,sinks", [(4000, 0), (5950, 100), (64, 64 * 90), (10 ** 6, 4)])
def test_wide_prefixes_behind_windows(window, sinks):
    _announce("shared wide window", window, sinks)
    lens = [6000 + t for t in (0, 1, 63, 64, 700, 2000, 30, 5)]
    g = Groups([(8, 6000)], lens, 1, 64, 32, "bf16", seed=15)
    g.run_and_check(256, "bf16", seed=15, window=window, sinks=sinks, rows=[0, 1, 4, 5])
    g.b.table[0, 20] = -1                    # a page that is gone, and one that was never of the pool
    g.b.table[0, 180] = 10 ** 7
    g.run_and_check(256, "bf16", seed=15, window=window, sinks=sinks, rows=[0, 3, 5])


@pytest.mark.parametrize("dtype,io", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f32")])
def test_wide_prefixes_with_values_that_are_not_finite(dtype, io):
    _announce("shared wide infinite", dtype, io)
    prefix = 9000
    g = Groups([(9, prefix)], [prefix + t for t in (0, 3, 64, 200, 1, 2, 3, 4, 5)], 1, 64, 32, dtype, seed=16)
    b = g.b
    for s, at, ch, x in ((0, 3, 1, INF), (0, 5000, 2, -INF), (0, 8999, 0, NAN), (0, 100, 5, INF), (0, 7000, 5, -INF), (1, prefix + 1, 3, INF),
                         (3, prefix + 150, 2, INF), (3, prefix + 151, 60, -INF)):
        b.v[s][at, 0, ch] = x
    g.write()
    g.run_and_check(256, io, seed=16, scale=0.1, rows=[0, 1, 2, 3, 8])
    k, v, table, lens = b.on(DEV)            # what lies behind the prefix and in other pages changes no bit
    q = torch.randn(9, 256 * 64, generator=torch.Generator().manual_seed(1)).to(M.DTYPES[io]).to(DEV)
    outs = []
    for fill in (0.0, INF, 3.0):
        v2 = v.clone()
        spare = [i for i in range(b.pages) if not bool((b.table == i).any())]
        v2[spare] = fill
        outs.append(g.run(256, q, 0.1, tensors=(k, v2, table, lens)))
    assert all(torch.equal(torch.nan_to_num(o, 7.0, 8.0, 9.0), torch.nan_to_num(outs[0], 7.0, 8.0, 9.0)) for o in outs)


def test_a_wide_prefix_among_more_sequences_than_a_launch_takes():
    """A group on both sides of the 1024th sequence whose prefix is wide in either launch."""
    _announce("shared wide 1100 sequences")
    prefix = 5000
    groups = [(900, 20), (200, prefix)]
    lens = [20 + i % 7 for i in range(900)] + [prefix + i % 9 for i in range(200)]
    Groups(groups, lens, 1, 64, 32, "bf16", seed=17).run_and_check(16, "bf16", seed=17, rows=[0, 899, 900, 1000, 1023, 1024, 1025, 1099])


def test_more_sequences_than_a_launch_takes():
    """Groups that lie on both sides of the 1024th sequence, and one of more than that."""
    _announce("shared 2500 sequences")
    groups = [(1000, 40), (100, 70), (0, 3), (1390, 33), (10, 0)]
    lens = [p + (37 * i) % 50 for m, p in groups for i in range(m)]
    Groups(groups, lens, 1, 64, 32, "bf16", seed=4, width=5).run_and_check(
        2, "f32", seed=4, rows=[0, 1, 999, 1000, 1001, 1023, 1024, 1025, 1099, 1100, 2047, 2048, 2489, 2490, 2499])


def test_members_shorter_than_the_prefix():
    _announce("shared short members")
    g = Groups([(4, 100), (3, 64)], [130, 40, 0, 100, 64, 90, 30], 2, 64, 16, "bf16", seed=5)
    g.run_and_check(4, "f32", seed=5)
    g.run_and_check(4, "f32", seed=5, window=30, sinks=3)
    # the first members, too: their pages hold the prefix all the same
    g.b.lens[0], g.b.lens[4] = 50, 20
    g.b.k[0], g.b.v[0], g.b.k[4], g.b.v[4] = g.b.k[0][:50], g.b.v[0][:50], g.b.k[4][:20], g.b.v[4][:20]
    g.b.kv_len = torch.tensor(g.b.lens, dtype=torch.int32)
    g.run_and_check(4, "f32", seed=5)


def test_missing_pages_and_bad_lengths():
    _announce("shared missing pages")
    g = Groups([(3, 128), (2, 96)], [200, 220, 129, 300, 128], 2, 64, 32, "bf16", seed=6)
    b = g.b
    b.table[0, 1] = -1                       # of the prefix: for all three
    b.table[1, 5] = 10 ** 6                  # of the second's own tokens
    b.table[3, 0] = -2 ** 31
    g.run_and_check(4, "f32", seed=6)
    k, v, table, lens = b.on(DEV)
    lens[1], lens[4] = -5, 10 ** 9           # lengths that no row of the table holds: what it holds counts
    start, prefix = g.arrays()
    q = torch.randn(5, 256, device=DEV)
    out = g.run(4, q, 0.125, tensors=(k, v, table, lens))
    assert not out[1].any() and bool(torch.isfinite(out[4]).all())
    prefix[0], prefix[1] = -7, 2 ** 31 - 1   # no prefix at all; all of the row
    out = g.run(4, q, 0.125, tensors=b.on(DEV), arrays=(start, prefix)).cpu().view(5, 4, 64)
    seen = ((b.table[0] >= 0) & (b.table[0] < b.pages))[torch.arange(200) // 32][None]
    want, tol = M.attention(q[0].cpu().view(1, 4, 64), b.k[0], b.v[0], seen, 0.125, M.io_eps("f32"), 0.0)
    M.check(out[0][None], want, tol, "a negative prefix is none")
    # the fourth row alone: the fifth sees its first 128 keys
    seen = ((b.table[3] >= 0) & (b.table[3] < b.pages))[torch.arange(128) // 32][None]
    want, tol = M.attention(q[4].cpu().view(1, 4, 64), b.k[3][:128], b.v[3][:128], seen, 0.125, M.io_eps("f32"), 0.0)
    M.check(out[4][None], want, tol, "a prefix past the table")


def test_rows_that_no_group_owns_stay():
    _announce("shared offsets")
    g = Groups([(2, 40), (3, 33)], [50, 60, 70, 33, 35], 1, 64, 16, "f16", seed=7)
    q = torch.randn(5, 128, generator=torch.Generator().manual_seed(7))
    i32 = dict(dtype=torch.int32, device=DEV)
    whole = g.run(2, q.to(DEV), 0.1).cpu()
    for start, owned in (([2, 5], [2, 3, 4]), ([0, 2], [0, 1]), ([0, 2, 2, 4], [0, 1, 2, 3]), ([0, 2, 9], [0, 1]), ([-3, 2, 5], [2, 3, 4]), ([5, 2, 5], [2, 3, 4])):
        prefix = {2: 33, 0: 40}
        lens = [prefix.get(s, 0) for s in start[:-1]]
        out = g.run(2, q.to(DEV), 0.1, arrays=(torch.tensor(start, **i32), torch.tensor(lens, **i32)), fill=7.0).cpu()
        for s in range(5):
            if s in owned:
                assert bool(((out[s] - whole[s]).abs() < 1e-4).all()), (start, s)
            else:
                assert bool((out[s] == 7.0).all()), (start, s)


@pytest.mark.parametrize("io", ["f32", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D,page", [(4, 1, 64, 16), (6, 2, 100, 64), (8, 2, 128, 32), (17, 1, 256, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 20)])
def test_values_that_are_not_finite(H, Hkv, D, page, dtype, io, window, sinks):
    """In the prefix (seen by all, or by the one whose window reaches them) and in the members' own tokens."""
    _announce("shared infinite", H, Hkv, D, page, dtype, io, window)
    groups, lens = [(3, 100), (2, 3000), (1, 0), (4, 64)], [101, 130, 300, 3001, 3100, 70, 64, 80, 64, 200]
    g = Groups(groups, lens, Hkv, D, page, dtype, seed=D)
    b = g.b
    for s, at, ch, x in ((0, 3, 1, INF), (0, 70, 2, -INF), (0, 99, 0, NAN), (1, 110, 3, INF), (1, 112, 3, -INF), (2, 250, 4, -INF), (3, 0, 5, INF),
                         (3, 2500, 6, NAN), (3, 2990, 7, -INF), (4, 3050, 7, INF), (5, 1, 1, INF), (6, 63, 9, INF), (7, 64, 9, -INF), (9, 190, D - 1, NAN)):
        b.v[s][at, at % Hkv, ch] = x
    g.write()
    g.run_and_check(H, dtype if io == "cache" else io, seed=8, window=window, sinks=sinks, scale=0.1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_keys_that_are_not_finite(dtype):
    """A key whose score is -inf has no weight, one of +inf or NaN spoils the heads that see it."""
    _announce("shared infinite keys", dtype)
    g = Groups([(2, 64), (2, 40)], [100, 90, 41, 60], 1, 64, 16, dtype, seed=9)
    b = g.b
    b.k[0][5, 0, 0] = -INF                   # q is positive: -inf
    b.k[1][80, 0, 3] = -INF
    b.k[2][7, 0, 1] = INF
    b.k[3][50, 0, 1] = NAN
    g.write()
    q = torch.rand(4, 128, generator=torch.Generator().manual_seed(9)) + 0.1
    out = g.run(2, q.to(DEV), 0.125).cpu()
    assert bool(torch.isnan(out[2:]).all()) and bool(torch.isfinite(out[:2]).all())
    for s, gone in ((0, [5]), (1, [5, 80])):
        seen = torch.ones(1, b.lens[s], dtype=torch.bool)
        seen[0, gone] = False
        k = b.k[s].clone()
        k[gone] = 0.0
        want, tol = M.attention(q[s].view(1, 2, 64), k, b.v[s], seen, 0.125, M.io_eps("f32"), 0.0)
        M.check(out[s].view(1, 2, 64), want, tol, f"sequence {s}")


def test_what_is_not_seen_may_hold_anything():
    """Pages past the lengths, behind the window and of others hold infinities: no result changes a bit."""
    _announce("shared poison")
    g = Groups([(3, 70), (4, 200)], [75, 100, 71, 205, 300, 260, 201], 2, 128, 32, "bf16", seed=10)
    q = torch.randn(7, 8 * 128, device=DEV)
    for window, sinks in ((0, 0), (20, 3)):
        outs = []
        for fill in (0.0, INF, NAN):
            k, v, table, lens = g.b.on(DEV)
            k, v = (torch.where(torch.isnan(t), torch.full_like(t, fill), t) for t in (k, v))
            outs.append(g.run(8, q, 0.09, window, sinks, tensors=(k, v, table, lens)))
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_the_same_call_gives_the_same_bits_on_any_stream():
    _announce("shared streams")
    g = Groups([(10, 3000), (3, 500)], [3000 + 91 * i for i in range(10)] + [600, 501, 777], 2, 128, 64, "bf16", seed=11)
    q = torch.randn(13, 8 * 128, device=DEV)
    a = g.run(8, q, 0.09)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        assert torch.equal(a, g.run(8, q, 0.09, stream=side))


def test_agrees_with_decode_of_single_sequences():
    """Groups of one sequence without a prefix are bitnet_attn_decode, whatever part of a sequence is called its prefix."""
    _announce("shared against decode")
    lens = [1, 70, 500, 3000]
    b = M.Batch(lens, 2, 128, 32, "bf16", seed=12)
    q = torch.randn(4, 8 * 128, device=DEV)
    k, v, table, kv_len = b.on(DEV)
    want = torch.empty_like(q)
    ws = torch.empty(max(16, B.bitnet_attn_decode_workspace_bytes(4, 8, 2, 128, 32, table.shape[1])), dtype=torch.uint8, device=DEV)
    B.bitnet_attn_decode(q, k, v, table, kv_len, want, 0.09, ws=ws)
    for prefix in ([0, 0, 0, 0], [1, 33, 500, 2999], [5, 70, 16, 10 ** 6]):
        g = Groups([(1, 0)] * 4, lens, 2, 128, 32, "bf16", seed=12)
        start = torch.arange(5, dtype=torch.int32, device=DEV)
        got = g.run(8, q, 0.09, arrays=(start, torch.tensor(prefix, dtype=torch.int32, device=DEV)), tensors=(k, v, table, kv_len))
        # both are within (D + 16 + n + 64) 2^-22 of the definition, relative to sums of |p v| <= 6 here
        assert float((got - want).abs().max()) < 2 * 6 * (144 + 3064) * 2.0 ** -22


def test_binding_refusals():
    b = M.Batch([4, 4], 2, 64, 16, "bf16", seed=1)
    k, v, table, kv_len = b.on(DEV)
    q = torch.zeros(2, 256, device=DEV)
    i = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    ws = torch.empty(B.bitnet_attn_decode_shared_workspace_bytes(2, 4, 2, 64, 16, table.shape[1]) + 16, dtype=torch.uint8, device=DEV)
    for kw, err in ((dict(group_start=i(0, 2, 2)), ValueError), (dict(q=q[:1], out=q[:1]), ValueError), (dict(prefix_len=i(3).long()), TypeError),
                    (dict(out=q.half()), ValueError), (dict(q=q.cpu(), out=q.cpu()), TypeError), (dict(group_start=i(0, 1, 1, 2), prefix_len=i(1, 1, 1)), B.BitnetError)):
        a = dict(q=q, group_start=i(0, 2), prefix_len=i(3), k_cache=k, v_cache=v, table=table, kv_len=kv_len, out=torch.empty_like(q), scale=1.0, ws=ws)
        a.update(kw)
        with pytest.raises(err):
            B.bitnet_attn_decode_shared(**a)
    out = torch.full_like(q, 3.0)
    B.bitnet_attn_decode_shared(q, i(0), i(), k, v, table, kv_len, out, 1.0, ws=ws)     # no groups: nothing written
    assert bool((out == 3.0).all())


def test_pages_past_four_gib():
    """The same pages at the lowest and at the highest numbers of a pool of 5 GiB of keys and as much of values, for prefixes in
    registers and in shared memory: the same bits; and tokens appended there."""
    _announce("shared pages past 4 GiB")
    Hkv, D, page, pages = 8, 128, 256, 10300
    k = torch.empty(pages, Hkv, D // 8, page, 8, dtype=torch.bfloat16, device=DEV)
    v = torch.empty(pages, Hkv, page // 8, D, 8, dtype=torch.bfloat16, device=DEV)
    assert k.numel() * 2 > 5 << 30
    g = torch.Generator(device=DEV).manual_seed(5)
    used = 90
    k[:used].copy_(torch.randn(used, *k.shape[1:], device=DEV, generator=g))
    v[:used].copy_(torch.randn(used, *v.shape[1:], device=DEV, generator=g))
    high = pages - 1 - torch.arange(used, device=DEV)
    k[high], v[high] = k[:used].clone(), v[:used].clone()
    i32 = dict(dtype=torch.int32, device=DEV)
    for prefix, H in ((700, 16), (20000, 256)):
        first = -(-prefix // page)
        rows = [list(range(first)) + [first + 2 * s, first + 2 * s + 1] for s in range(4)]
        lens = torch.tensor([first * page + 10 + 70 * s for s in range(4)], **i32)
        q = torch.randn(4, H * D, device=DEV, generator=g).to(torch.bfloat16)
        outs = []
        for ids in (torch.arange(used, device=DEV), high):
            table = ids[torch.tensor(rows, device=DEV)].to(torch.int32).contiguous()
            out = torch.empty_like(q)
            ws = torch.empty(B.bitnet_attn_decode_shared_workspace_bytes(4, H, Hkv, D, page, table.shape[1]), dtype=torch.uint8, device=DEV)
            B.bitnet_attn_decode_shared(q, torch.tensor([0, 4], **i32), torch.tensor([prefix], **i32), k, v, table, lens, out, 0.09, ws=ws)
            outs.append(out)
        assert torch.equal(*outs) and bool(torch.isfinite(outs[0]).all()), prefix
    freqs = torch.empty(64, dtype=torch.float64, device=DEV)
    B.bitnet_rope_freqs(freqs, 10000.0)
    kn, vn = torch.randn(20, Hkv * D, device=DEV, generator=g), torch.randn(20, Hkv * D, device=DEV, generator=g)
    lens, start = torch.tensor([520], **i32), torch.tensor([0, 20], **i32)
    for ids in (torch.arange(3, device=DEV), high[:3]):
        B.bitnet_kv_append_rope(kn, vn, start, k, v, ids[None].to(torch.int32).contiguous(), lens, freqs)
    assert torch.equal(k[:3], k[high[:3]]) and torch.equal(v[:3], v[high[:3]])
    assert torch.equal(v[2, :, 0, :, 0].reshape(-1), vn[12].to(torch.bfloat16))     # position 512 is the third page's first
