"""Plain 64-bit models of the paged cache's calls, on the CPU: cache layout, attention, and the page tables."""
from __future__ import annotations

import math

import torch

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


class Batch:
    """Sequences of given lengths with random keys and values, their page table and caches.  Every element of the caches
    that belongs to no token holds `fill` (NaN by default): nothing may read it into a result."""

    def __init__(self, lens, heads, dim, page, dtype, seed, spare=2, fill=float("nan"), width=None):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.heads, self.dim, self.page, self.dtype = list(lens), heads, dim, page, DTYPES[dtype]
        need = [-(-n // page) for n in self.lens]
        self.pages = sum(need) + spare
        self.width = width if width is not None else max(need + [0]) + 1
        ids = torch.randperm(self.pages, generator=g)
        self.table = torch.full((len(self.lens), self.width), -1, dtype=torch.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = ids[at:at + n].to(torch.int32)
            at += n
        self.chunks = -(-dim // 8)
        self.k_cache = torch.full((self.pages, heads, self.chunks, page, 8), fill, dtype=self.dtype)
        self.v_cache = torch.full((self.pages, heads, page // 8, dim, 8), fill, dtype=self.dtype)
        self.k = [torch.randn(n, heads, dim, generator=g).to(self.dtype) for n in self.lens]
        self.v = [torch.randn(n, heads, dim, generator=g).to(self.dtype) for n in self.lens]
        for s in range(len(self.lens)):
            self.write(s, 0, self.k[s], self.v[s])
        self.kv_len = torch.tensor(self.lens, dtype=torch.int32)

    def write(self, s, first, k, v):
        pos = torch.arange(first, first + k.shape[0])
        page, slot = self.table[s][pos // self.page].long(), pos % self.page
        pad = torch.zeros(k.shape[0], self.heads, self.chunks * 8 - self.dim, dtype=k.dtype)
        self.k_cache[page, :, :, slot] = torch.cat([k, pad], 2).view(k.shape[0], self.heads, self.chunks, 8)
        self.v_cache[page, :, slot // 8, :, slot % 8] = v

    def on(self, dev):
        return [t.to(dev) for t in (self.k_cache, self.v_cache, self.table, self.kv_len)]


def visible(pos, keys, window, n_sink):
    """[len(pos), keys] truth values: does the query at each position see key j?"""
    j, p = torch.arange(keys)[None, :], pos[:, None]
    near = j <= p
    return near & ((j > p - window) | (j < n_sink)) if window else near


def attention(q, k, v, seen, scale, io_eps, weight_eps):
    """(out, tolerance) in 64 bits of q [n, H, D] over k, v [L, Hkv, D]; seen [n, L].  Keys that are not seen do not enter.

    The tolerance follows the arithmetic: a score is a sum of D products in 32 bits (u = 2^-22 an addition: the matrix
    instruction may round its partial sums more coarsely than a single addition does), the exponent takes its error as a
    relative one, the weighted sum and its divisor add L + 64 roundings more; weight_eps is the rounding of a weight to the
    cache's type (0 where it stays in parts), io_eps that of the output."""
    n, H, D = q.shape
    G = H // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, tol = torch.zeros(n, H, D, dtype=torch.float64), torch.zeros(n, H, D, dtype=torch.float64)
    u = 2.0 ** -22
    some = seen.any(1)
    for h in range(H):
        kh, vh = k[:, h // G], v[:, h // G]
        x = scale * (q[:, h] @ kh.t())
        size = abs(scale) * (q[:, h].abs() @ torch.nan_to_num(kh, 0.0, 0.0, 0.0).abs().t())
        x = x.masked_fill(~seen, -math.inf)
        x[~some] = 0.0
        p = torch.softmax(x, 1).masked_fill(~seen, 0.0)
        clean = torch.isfinite(vh)
        o = p @ torch.where(clean, vh, 0.0)
        for j, d in (~clean).nonzero().tolist():          # values that are not finite, where they are seen
            o[seen[:, j], d] += vh[j, d]
        out[:, h] = o
        score = ((D + 16) * u * size + 4 * u * x.abs().masked_fill(~seen, 0.0)).masked_fill(~seen, 0.0).amax(1, keepdim=True)
        mass = p @ torch.where(clean, vh, 0.0).abs()
        tol[:, h] = (2 * score + (k.shape[0] + 64) * u + weight_eps) * mass + io_eps * torch.nan_to_num(o, 0.0, 0.0, 0.0).abs() + 1e-30
    return out, tol


def check(got, want, tol, what=""):
    got = got.detach().double().cpu()
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{what}: finite values differ"
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    assert bool(same[~finite].all()), f"{what}: values that are not finite differ"
    err = (got - want).abs()[finite]
    bad = err > tol[finite]
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {err.numel()} outside, worst {float((err / tol[finite]).max())} of the tolerance"


def io_eps(io):
    return {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}[io]


# ---------------------------------------------------------------------------------------------------------------------
# Page tables as plain lists
# ---------------------------------------------------------------------------------------------------------------------
class Pages:
    """table, kv_len and refs of a pool, and what every page holds (a label that copying carries along)."""

    def __init__(self, n_seqs, width, n_pages, page):
        self.page, self.width, self.n_pages = page, width, n_pages
        self.table = [[-1] * width for _ in range(n_seqs)]
        self.lens = [0] * n_seqs
        self.refs = [0] * n_pages
        self.holds = list(range(n_pages))

    def free_ids(self):
        return [i for i, r in enumerate(self.refs) if r == 0]

    def reserve(self, seqs, n_new):
        free, at, short = self.free_ids(), 0, 0
        for s, n in zip(seqs, n_new):
            if not 0 <= s < len(self.lens) or n < 0 or self.lens[s] + n > self.width * self.page:
                short += 1
                continue
            first, last = -(-self.lens[s] // self.page), -(-(self.lens[s] + n) // self.page)
            take, at = free[at:at + last - first], at + last - first
            if len(take) < last - first:
                short += 1
                continue
            for j, p in enumerate(take):
                self.table[s][first + j] = p
                self.refs[p] = 1
            self.lens[s] += n
        return short

    def fork(self, parents, children):
        free, at, short = self.free_ids(), 0, 0
        n = len(self.lens)
        for p, c in zip(parents, children):
            if not (0 <= p < n and 0 <= c < n) or p == c:
                short += 1
                continue
            full, rest = divmod(self.lens[p], self.page)
            row = self.table[p][:full] + [-1] * (self.width - full)
            if rest and self.table[p][full] >= 0:
                if at >= len(free):
                    at += 1
                    short += 1
                    self.table[c], self.lens[c] = [-1] * self.width, 0
                    continue
                row[full] = free[at]
                self.holds[free[at]] = self.holds[self.table[p][full]]
                self.refs[free[at]] = 1
                at += 1
            for e in row[:full]:
                if e >= 0:
                    self.refs[e] += 1
            self.table[c], self.lens[c] = row, self.lens[p]
        return short

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.lens):
                for e in self.table[s]:
                    if e >= 0:
                        self.refs[e] -= 1
                self.table[s], self.lens[s] = [-1] * self.width, 0

    def trim(self, seqs, window, n_sink):
        for s in seqs:
            for t in range(self.width):
                lo, hi = t * self.page, (t + 1) * self.page
                if lo >= n_sink and hi <= self.lens[s] + 1 - window and self.table[s][t] >= 0:
                    self.refs[self.table[s][t]] -= 1
                    self.table[s][t] = -1

    def compact(self):
        live = [i for i, r in enumerate(self.refs) if r > 0]
        n = len(live)
        holes = [i for i in range(n) if self.refs[i] == 0]
        moved = dict(zip([i for i in reversed(live) if i >= n], holes))
        for src, dst in moved.items():
            self.holds[dst] = self.holds[src]
            self.refs[dst], self.refs[src] = self.refs[src], 0
        self.table = [[moved.get(e, e) for e in row] for row in self.table]
        return n
