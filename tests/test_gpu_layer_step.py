"""The calls between a layer's products together, as a serving loop makes them: norm and codes, q/k/v, rotation and append, decode over
a shared prefix, norm and codes, o.  Eager, on a side stream, and captured into a graph that is replayed with other inputs
and positions; against the separate calls and against plain operations."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from paper_2502_11880_amd import inputs
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HIDDEN, HEADS, KV, DIM, PAGE, PREFIX, SEQS, WIDTH = 512, 8, 2, 64, 16, 150, 6, 20
EPS = 1e-5


def _pack(n, k, seed):
    w = inputs.weight_f32(n, k, seed=inputs.seed_for(0, seed)).to(DEV)
    p, s = torch.empty(B.bitnet_packed_bytes("i2s", n, k), dtype=torch.uint8, device=DEV), torch.empty(1, device=DEV)
    B.bitnet_pack_weights("i2s", w, p, s, torch.empty(B.bitnet_pack_workspace_bytes(n, k), dtype=torch.uint8, device=DEV))
    return p, s


class Layer:
    """Three sequences that share a prefix and three of their own, one more token each a step."""

    def __init__(self):
        e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=DEV)  # noqa: E731
        self.packs = [_pack(n, HIDDEN, 50 + i) for i, n in enumerate((HEADS * DIM, KV * DIM, KV * DIM))]
        self.o_pack = _pack(HIDDEN, HEADS * DIM, 60)
        g = torch.Generator(device=DEV).manual_seed(3)
        self.gamma, self.gamma2 = (1 + 0.2 * torch.randn(n, device=DEV, generator=g) for n in (HIDDEN, HEADS * DIM))
        lens = [PREFIX + t for t in (1, 20, 75)] + [33, 1, 90]
        b = M.Batch(lens, KV, DIM, PAGE, "bf16", seed=21, fill=0.0, spare=30, width=WIDTH)
        spare = [i for i in range(b.pages) if not bool((b.table == i).any())]
        for s in range(SEQS):                    # room for the next tokens
            b.table[s, -(-lens[s] // PAGE):-(-lens[s] // PAGE) + 2] = torch.tensor([spare.pop(), spare.pop()])
        for s in (1, 2):                         # whole pages of the prefix are the first one's
            b.table[s, :PREFIX // PAGE] = b.table[0, :PREFIX // PAGE]
        self.k, self.v, self.table, self.kv_len = b.on(DEV)
        low = PREFIX // PAGE * PAGE              # and the page that it ends in is copied
        for s in (1, 2):
            src, dst = int(b.table[0, PREFIX // PAGE]), int(b.table[s, PREFIX // PAGE])
            self.k[dst, :, :, :PREFIX - low] = self.k[src, :, :, :PREFIX - low]
            for t in range(PREFIX - low):
                self.v[dst, :, t // 8, :, t % 8] = self.v[src, :, t // 8, :, t % 8]
        self.k0, self.v0, self.len0 = self.k.clone(), self.v.clone(), self.kv_len.clone()
        self.groups = torch.tensor([0, 3, 4, 5, 6], dtype=torch.int32, device=DEV)
        self.prefix = torch.tensor([PREFIX, 0, 0, 0], dtype=torch.int32, device=DEV)
        self.freqs = e(DIM // 2, t=torch.float64)
        B.bitnet_rope_freqs(self.freqs, 10000.0, "turns", 4.0, 64, 1.0, 4.0)
        self.h, self.res = e(SEQS, HIDDEN), e(SEQS, HIDDEN, t=torch.bfloat16)
        self.xq, self.xs, self.rs = e(SEQS, HIDDEN, t=torch.int8), e(SEQS), e(SEQS, t=torch.int32)
        self.aq, self.asc, self.ars = e(SEQS, HEADS * DIM, t=torch.int8), e(SEQS), e(SEQS, t=torch.int32)
        self.q, self.kn, self.vn = e(SEQS, HEADS * DIM), e(SEQS, KV * DIM), e(SEQS, KV * DIM)
        self.attn, self.out = e(SEQS, HEADS * DIM), e(SEQS, HIDDEN)
        self.ws = e(max(16, B.bitnet_attn_decode_shared_workspace_bytes(SEQS, HEADS, KV, DIM, PAGE, WIDTH)), t=torch.uint8)
        self.one = torch.ones(SEQS, dtype=torch.int32, device=DEV)

    def reset(self, h, res):
        self.k.copy_(self.k0)
        self.v.copy_(self.v0)
        self.kv_len.copy_(self.len0)
        self.h.copy_(h)
        self.res.copy_(res)

    def step(self):
        self.kv_len.add_(self.one)
        B.bitnet_norm_quantize(self.h, self.gamma, EPS, self.xq, self.xs, self.rs, self.res, self.res)
        B.bitnet_mpgemm_fused("i2s", [p for p, _ in self.packs], [s for _, s in self.packs], None, self.xq, self.xs, self.rs, [self.q, self.kn, self.vn])
        B.bitnet_kv_append_rope(self.kn, self.vn, None, self.k, self.v, self.table, self.kv_len, self.freqs, q=self.q, q_out=self.q)
        B.bitnet_attn_decode_shared(self.q, self.groups, self.prefix, self.k, self.v, self.table, self.kv_len, self.attn, 1 / math.sqrt(DIM), ws=self.ws)
        B.bitnet_norm_quantize(self.attn, self.gamma2, EPS, self.aq, self.asc, self.ars)
        B.bitnet_mpgemm_fused("i2s", [self.o_pack[0]], [self.o_pack[1]], None, self.aq, self.asc, self.ars, [self.h])

    def state(self):
        return [t.clone() for t in (self.h, self.res, self.q, self.attn, self.aq, self.k, self.v, self.kv_len)]

    def apart(self):
        """The same step by the calls that were there before, and plain operations between them."""
        self.kv_len.add_(self.one)
        self.res.copy_((self.h + self.res.float()).to(torch.bfloat16))
        r = self.res.float()
        n = r * (1 / torch.sqrt((r.double() ** 2).mean(1, keepdim=True) + torch.tensor(EPS).double())).float() * self.gamma
        ws = torch.empty(max(16, B.bitnet_mpgemm_fused_workspace_bytes("i2s", [HEADS * DIM, KV * DIM, KV * DIM], HIDDEN, SEQS)), dtype=torch.uint8, device=DEV)
        B.bitnet_mpgemm_fused("i2s", [p for p, _ in self.packs], [s for _, s in self.packs], n, self.xq, self.xs, self.rs, [self.q, self.kn, self.vn], ws)
        pos = (self.kv_len - 1).contiguous()
        B.bitnet_rope(self.q, pos, self.freqs, self.q, DIM)
        B.bitnet_rope(self.kn, pos, self.freqs, self.kn, DIM)
        B.bitnet_kv_append(self.kn, self.vn, None, self.k, self.v, self.table, self.kv_len)
        dec = torch.empty(max(16, B.bitnet_attn_decode_workspace_bytes(SEQS, HEADS, KV, DIM, PAGE, WIDTH)), dtype=torch.uint8, device=DEV)
        B.bitnet_attn_decode(self.q, self.k, self.v, self.table, self.kv_len, self.attn, 1 / math.sqrt(DIM), ws=dec)
        return n


def _inputs(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(SEQS, HIDDEN, device=DEV, generator=g), torch.randn(SEQS, HIDDEN, device=DEV, generator=g).to(torch.bfloat16)


def test_a_step_is_the_separate_calls():
    print("case: layer step", flush=True)
    layer, apart = Layer(), Layer()
    for x in (layer, apart):
        x.reset(*_inputs(1))
        for _ in range(3):                       # two steps that leave the state alike, then the compared one
            h, res = _inputs(2)
            x.h.copy_(h)
            x.res.copy_(res)
            x.step() if x is layer else x.apart()
    for name in ("res", "xq", "xs", "rs", "q", "k", "v", "kv_len"):
        assert torch.equal(getattr(layer, name), getattr(apart, name)), name
    # the attention adds up in another order: both within (D + 16 + n + 64) 2^-22 of sums of |p v| <= max |v|
    assert float((layer.attn - apart.attn).abs().max()) <= 2 * (DIM + 16 + 230 + 64) * 2.0 ** -22 * float(layer.v.float().abs().max())


def test_steps_in_a_graph_and_on_another_stream():
    """Replays with other inputs, cache contents and lengths than the captured ones, eager work between them."""
    print("case: layer step in a graph", flush=True)
    layer = Layer()
    want = []
    for seed in range(4):
        layer.reset(*_inputs(seed))
        if seed == 3:
            layer.kv_len[4] = 25                 # of pages that are not there, too
        layer.step()
        layer.step()
        want.append(layer.state())
    layer.reset(*_inputs(9))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        layer.step()
        with torch.cuda.graph(graph, stream=side):
            layer.step()
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        for seed in range(4):
            layer.reset(*_inputs(seed))
            if seed == 3:
                layer.kv_len[4] = 25
            graph.replay()
            if turn == 1:
                torch.cuda.synchronize()
            graph.replay()
            for a, b in zip(layer.state(), want[seed]):
                assert torch.equal(a, b), (turn, seed)
    with torch.cuda.stream(side):                # eager, on that stream
        layer.reset(*_inputs(0))
        layer.step()
        layer.step()
        got = layer.state()
    side.synchronize()
    for a, b in zip(got, want[0]):
        assert torch.equal(a, b)


def test_calls_at_once_on_two_streams():
    """Two layers, each with its workspace, on two streams: the results of either alone."""
    print("case: two layers at once", flush=True)
    layers = [Layer(), Layer()]
    want = []
    for i, x in enumerate(layers):
        x.reset(*_inputs(i))
        for _ in range(5):
            x.step()
        want.append(x.state())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for i, (x, s) in enumerate(zip(layers, streams)):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            x.reset(*_inputs(i))
    for _ in range(5):
        for x, s in zip(layers, streams):
            with torch.cuda.stream(s):
                x.step()
    torch.cuda.synchronize()
    for x, w in zip(layers, want):
        for a, b in zip(x.state(), w):
            assert torch.equal(a, b)
