"""Values and keys that are not finite where a query does see them, against the definition: a value of +inf or -inf makes its
channel that infinity (both, or a NaN: NaN) whatever its weight and wherever its tile, split or joined; a key whose score is
-inf has no weight."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
INF, NAN = float("inf"), float("nan")


def _announce(*what):
    print("case:", *what, flush=True)


def _decode(b, H, q, scale, window=0, sinks=0):
    k, v, table, lens = b.on(DEV)
    out = torch.full_like(q, 7.0)
    need = B.bitnet_attn_decode_workspace_bytes(len(b.lens), H, b.heads, b.dim, b.page, table.shape[1], window, sinks)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    B.bitnet_attn_decode(q, k, v, table, lens, out, scale, window, sinks, ws)
    torch.cuda.synchronize()
    return out.cpu().view(-1, H, b.dim)


def _prefill(b, H, q, new, scale, window=0, sinks=0, split=True):
    k, v, table, lens = b.on(DEV)
    start = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).to(DEV)
    out = torch.full_like(q, 7.0)
    B.bitnet_attn_prefill(q, start, k, v, table, lens, out, scale, window, sinks,
                          ws=None if split else torch.empty(16, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    return out.cpu().view(-1, H, b.dim)


def _plant(v, at):
    """Values that are not finite in a sequence's v [L, Hkv, D], around position `at`."""
    n, d = v.shape[0], v.shape[2]
    for i, (channel, values) in enumerate({0: [INF], 1: [-INF], 2: [INF, -INF], 3: [NAN], d // 2: [INF, INF], d - 1: [NAN, INF]}.items()):
        for j, x in enumerate(values):
            v[(at + 3 * i + j) % n, i % v.shape[1], channel] = x


@pytest.mark.parametrize("io", ["f32", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D,page", [(4, 1, 64, 16), (6, 2, 100, 64), (8, 2, 128, 32), (17, 1, 256, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 20)])
def test_decode_values_that_are_seen(H, Hkv, D, page, dtype, io, window, sinks):
    _announce("decode infinite values", H, Hkv, D, page, dtype, io, window)
    b = M.Batch([1, 33, 90, 300, 700, 5000], Hkv, D, page, dtype, seed=D)
    b.v[0][0, 0, 1] = INF                    # a weight of exactly 1: its later parts are 0
    for s, at in ((1, 3), (2, 70), (3, 1), (4, 690), (5, 2500)):
        _plant(b.v[s], at)
    if window:
        b.v[5][4000, 0, 5] = INF             # behind the window, and past the sinks: not seen
        b.v[5][7, 0, 6] = -INF               # a sink
    for s in range(6):
        b.write(s, 0, b.k[s], b.v[s])
    io = dtype if io == "cache" else io
    q = torch.randn(6, H * D, generator=torch.Generator().manual_seed(41)).to(M.DTYPES[io])
    out = _decode(b, H, q.to(DEV), 0.1, window, sinks)
    for s, n in enumerate(b.lens):
        seen = M.visible(torch.tensor([n - 1]), n, window, sinks)
        want, tol = M.attention(q[s].view(1, H, D), b.k[s], b.v[s], seen, 0.1, M.io_eps(io), 2.0 ** -15 if io != "f32" else 0.0)
        M.check(out[s][None], want, tol, f"sequence {s} of {n}")


def _towering(n, heads, D, dtype, seed, page, key):
    """A sequence whose key `key` has a score so far above the others' that their weights, and the factors that their parts
    are joined with, are 0 in 32 bits."""
    b = M.Batch([n], heads, D, page, dtype, seed=seed)
    b.k[0][key] = 60.0
    return b


@pytest.mark.parametrize("dtype,io", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("key", [5, 9000])
def test_decode_infinite_values_of_weights_that_vanish(dtype, io, key):
    _announce("decode infinite values of no weight", dtype, io, key)
    b = _towering(9001, 1, 64, dtype, 42, 64, key)
    b.v[0][4000, 0, 3] = INF
    b.v[0][4001, 0, 9] = -INF
    b.v[0][8990, 0, 11] = INF
    b.v[0][30, 0, 13] = NAN
    b.write(0, 0, b.k[0], b.v[0])
    q = torch.rand(1, 2 * 64, generator=torch.Generator().manual_seed(42)).to(M.DTYPES[io]) + 0.5
    out = _decode(b, 2, q.to(DEV), 0.2)
    want, tol = M.attention(q.view(1, 2, 64), b.k[0], b.v[0], torch.ones(1, 9001, dtype=torch.bool), 0.2, M.io_eps(io),
                            2.0 ** -15 if io != "f32" else 0.0)
    M.check(out, want, tol)


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("io", ["f32", "cache"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("H,Hkv,D,page", [(4, 1, 64, 16), (6, 2, 100, 64), (8, 2, 128, 32), (3, 1, 256, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (400, 20)])
def test_prefill_values_that_are_seen(H, Hkv, D, page, dtype, io, window, sinks, split):
    _announce("prompt infinite values", H, Hkv, D, page, dtype, io, window, split)
    new, past = [1, 130, 40], [0, 1000, 1700]
    b = M.Batch([n + p for n, p in zip(new, past)], Hkv, D, page, dtype, seed=D + 1)
    b.v[0][0, 0, 1] = INF                    # a weight of exactly 1
    _plant(b.v[1], 900)                      # in tiles that every query sees whole
    _plant(b.v[2], 1300)
    b.v[1][1100, 0, 7] = INF                 # among the new tokens: seen by the later ones only
    b.v[2][3, 0, 9] = -INF                   # a sink, or behind the window
    for s in range(3):
        b.write(s, 0, b.k[s], b.v[s])
    io = dtype if io == "cache" else io
    weight = 0.0 if io == "f32" else {"bf16": 2.0 ** -8, "f16": 2.0 ** -10}[io]
    q = torch.randn(sum(new), H * D, generator=torch.Generator().manual_seed(43)).to(M.DTYPES[io])
    out = _prefill(b, H, q.to(DEV), new, 0.1, window, sinks, split)
    at = 0
    for s, n in enumerate(new):
        L = b.lens[s]
        want, tol = M.attention(q[at:at + n].view(n, H, D), b.k[s], b.v[s], M.visible(torch.arange(L - n, L), L, window, sinks), 0.1,
                                M.io_eps(io), weight)
        M.check(out[at:at + n], want, tol, f"sequence {s}")
        at += n


@pytest.mark.parametrize("split", [True, False])
@pytest.mark.parametrize("dtype,io", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("key", [5, 2990])
def test_prefill_infinite_values_of_weights_that_vanish(dtype, io, key, split):
    _announce("prompt infinite values of no weight", dtype, io, key, split)
    b = _towering(3000, 1, 64, dtype, 44, 64, key)
    b.v[0][1000, 0, 3] = INF
    b.v[0][1001, 0, 9] = -INF
    b.v[0][2950, 0, 11] = INF
    b.v[0][30, 0, 13] = NAN
    b.write(0, 0, b.k[0], b.v[0])
    q = torch.rand(70, 2 * 64, generator=torch.Generator().manual_seed(44)).to(M.DTYPES[io]) + 0.5
    weight = 0.0 if io == "f32" else {"bf16": 2.0 ** -8, "f16": 2.0 ** -10}[io]
    out = _prefill(b, 2, q.to(DEV), [70], 0.2, split=split)
    want, tol = M.attention(q.view(70, 2, 64), b.k[0], b.v[0], M.visible(torch.arange(2930, 3000), 3000, 0, 0), 0.2, M.io_eps(io), weight)
    M.check(out, want, tol)
