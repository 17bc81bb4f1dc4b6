"""The attention half of a ternary decoder layer, served from a paged cache.

    python examples/attention_layer.py

A prompt and then single tokens go through q/k/v (``bitnet_mpgemm_fused``), the cache (``bitnet_kv_reserve``,
``bitnet_kv_append``), the attention (``bitnet_attn_prefill``, ``bitnet_attn_decode``) and o.  After the prompt the sequence is
forked into two beams (``bitnet_kv_fork``); with a sliding window the pages behind it are given back as the beams grow
(``bitnet_kv_trim``); in the end one beam is freed and the pool compacted (``bitnet_kv_free``, ``bitnet_kv_compact``), and the
other goes on from where its pages now are.  Every attention output is checked against plain attention over all tokens so far.
The hidden states are random: the layer's other half, embeddings and positions are left out.
"""
from __future__ import annotations

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2502_11880_amd as B
from paper_2502_11880_amd import inputs

DEV = "cuda:0"


class Linears:
    """Weights that read one activation, packed I2_S, and the buffers of their products."""

    def __init__(self, weights):
        self.K = weights[0].shape[1]
        self.packed, self.scales, self.N = [], [], [w.shape[0] for w in weights]
        for w in weights:
            w = w.to(DEV)
            p = torch.empty(B.bitnet_packed_bytes("i2s", *w.shape), dtype=torch.uint8, device=DEV)
            s = torch.empty(1, device=DEV)
            B.bitnet_pack_weights("i2s", w, p, s, torch.empty(B.bitnet_pack_workspace_bytes(*w.shape), dtype=torch.uint8, device=DEV))
            self.packed.append(p)
            self.scales.append(s)

    def __call__(self, x):
        M = x.shape[0]
        xq, s = torch.empty(M, self.K, dtype=torch.int8, device=DEV), torch.empty(M, device=DEV)
        rowsum = torch.empty(M, dtype=torch.int32, device=DEV)
        ys = [torch.empty(M, n, device=DEV) for n in self.N]
        ws = torch.empty(max(16, B.bitnet_mpgemm_fused_workspace_bytes("i2s", self.N, self.K, M)), dtype=torch.uint8, device=DEV)
        B.bitnet_mpgemm_fused("i2s", self.packed, self.scales, x, xq, s, rowsum, ys, ws)
        return ys


class Layer:
    def __init__(self, hidden, heads, kv_heads, page=32, pages=64, max_pages=32, seqs=4, window=0, sinks=0, dtype=torch.bfloat16):
        self.heads, self.kv_heads, self.dim, self.page = heads, kv_heads, hidden // heads, page
        self.window, self.sinks, self.scale = window, sinks, 1 / math.sqrt(hidden // heads)
        kv = kv_heads * self.dim
        w = [inputs.weight_f32(n, hidden, seed=inputs.seed_for(0, 30 + i)) for i, n in enumerate((hidden, kv, kv, hidden))]
        self.qkv, self.o = Linears(w[:3]), Linears(w[3:])
        self.k_pool = torch.empty(1, pages, kv_heads, -(-self.dim // 8), page, 8, dtype=dtype, device=DEV)
        self.v_pool = torch.empty(1, pages, kv_heads, page // 8, self.dim, 8, dtype=dtype, device=DEV)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table, self.kv_len = torch.full((seqs, max_pages), -1, **i32), torch.zeros(seqs, **i32)
        self.refs, self.short = torch.zeros(pages, **i32), torch.zeros(1, **i32)
        self.ws = torch.empty(B.bitnet_kv_workspace_bytes(pages, seqs), dtype=torch.uint8, device=DEV)
        self.attn_ws = torch.empty(max(16, B.bitnet_attn_decode_workspace_bytes(seqs, heads, kv_heads, self.dim, page, max_pages,
                                                                                window, sinks)), dtype=torch.uint8, device=DEV)
        self.seen = {}                           # the plain copy that the outputs are checked against: rows of k and v

    def reserve(self, seqs, n_new):
        B.bitnet_kv_reserve(self.table, self.kv_len, self.refs, seqs, n_new, self.page, self.short, self.ws)

    def prompt(self, seq, x):
        """All tokens of a prompt as sequence `seq`."""
        n = x.shape[0]
        rows = slice(seq, seq + 1)
        ids = torch.tensor([seq], dtype=torch.int32, device=DEV)
        start = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        q, k, v = self.qkv(x)
        self.reserve(ids, torch.full_like(ids, n))
        B.bitnet_kv_append(k, v, start, self.k_pool[0], self.v_pool[0], self.table[rows], self.kv_len[rows])
        a = torch.empty_like(q)
        B.bitnet_attn_prefill(q, start, self.k_pool[0], self.v_pool[0], self.table[rows], self.kv_len[rows], a, self.scale,
                              self.window, self.sinks)
        self.seen[seq] = [k, v]
        self.check(a, q, [seq] * n, range(n))
        return self.o(a)[0]

    def step(self, first, count, x):
        """One more token for each of the sequences first .. first + count - 1."""
        rows = slice(first, first + count)
        ids = torch.arange(first, first + count, dtype=torch.int32, device=DEV)
        q, k, v = self.qkv(x)
        if self.window:
            B.bitnet_kv_trim(self.table, self.kv_len, self.refs, ids, self.page, self.window, self.sinks)
        self.reserve(ids, torch.ones_like(ids))
        B.bitnet_kv_append(k, v, None, self.k_pool[0], self.v_pool[0], self.table[rows], self.kv_len[rows])
        a = torch.empty_like(q)
        B.bitnet_attn_decode(q, self.k_pool[0], self.v_pool[0], self.table[rows], self.kv_len[rows], a, self.scale, self.window,
                             self.sinks, self.attn_ws)
        for i, s in enumerate(range(first, first + count)):
            self.seen[s] = [torch.cat([old, new[i:i + 1]]) for old, new in zip(self.seen[s], (k, v))]
        self.check(a, q, range(first, first + count), [self.seen[s][0].shape[0] - 1 for s in range(first, first + count)])
        return self.o(a)[0]

    def fork(self, parent, children):
        kids = torch.tensor(children, dtype=torch.int32, device=DEV)
        B.bitnet_kv_fork(self.k_pool, self.v_pool, self.table, self.kv_len, self.refs, torch.full_like(kids, parent), kids,
                         self.short, self.ws)
        for c in children:
            self.seen[c] = list(self.seen[parent])

    def free(self, seqs):
        B.bitnet_kv_free(self.table, self.kv_len, self.refs, torch.tensor(seqs, dtype=torch.int32, device=DEV))

    def compact(self):
        B.bitnet_kv_compact(self.k_pool, self.v_pool, self.table, self.refs, self.short, self.ws)
        return int(self.short)

    def check(self, a, q, seqs, positions):
        """Outputs a against plain attention in 64 bits over the tokens of each sequence, keys and values as the cache rounds
        them: within 1e-5 of the largest value."""
        for row, (s, p) in enumerate(zip(seqs, positions)):
            k, v = (t[:p + 1].to(self.k_pool.dtype).double().view(p + 1, self.kv_heads, self.dim) for t in self.seen[s])
            k, v = (t.repeat_interleave(self.heads // self.kv_heads, 1) for t in (k, v))
            x = (q[row].double().view(self.heads, 1, self.dim) * k.transpose(0, 1)).sum(-1) * self.scale
            if self.window:
                j = torch.arange(p + 1, device=DEV)
                x[:, (j <= p - self.window) & (j >= self.sinks)] = -math.inf
            want = (torch.softmax(x, -1)[..., None] * v.transpose(0, 1)).sum(1).reshape(-1)
            err = float((a[row].double() - want).abs().max() / want.abs().max())
            assert err < 1e-5, f"sequence {s}, position {p}: {err:.2g} off"


def main(window=0, sinks=0, hidden=1024, heads=8, kv_heads=2, prompt=150, steps=40):
    g = torch.Generator(device=DEV).manual_seed(1)
    hidden_states = lambda n: torch.randn(n, hidden, device=DEV, generator=g)  # noqa: E731
    layer = Layer(hidden, heads, kv_heads, window=window, sinks=sinks)
    layer.prompt(0, hidden_states(prompt))
    layer.fork(0, [1, 2])
    layer.free([0])
    for _ in range(steps):
        layer.step(1, 2, hidden_states(2))
    layer.free([1])
    live = layer.compact()
    assert live == int((layer.table[2] >= 0).sum()) and int(layer.table[2].max()) < live
    for _ in range(3):
        layer.step(2, 1, hidden_states(1))
    print(f"window {window}, sinks {sinks}: {prompt} + {steps} + 3 tokens, {live} live pages after compacting: every output checked", flush=True)


if __name__ == "__main__":
    main()
    main(window=64, sinks=4)
