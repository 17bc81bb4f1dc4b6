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


@pytest.mark.parametrize("dtype,io", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("scale", [0.1, -0.1])
@pytest.mark.parametrize("D", [64, 128, 100, 256])
def test_keys_whose_score_is_minus_infinity_have_no_weight(D, scale, dtype, io):
    """Channels of some keys are infinite; heads whose query has the sign that makes the score -inf leave them out, the others,
    whose score is +inf, become NaN."""
    _announce("infinite keys", D, scale, dtype, io)
    L, n, H, sign = 400, 50, 4, 1.0 if scale > 0 else -1.0
    b = M.Batch([L], 1, D, 32, dtype, seed=D + 2)
    bad = {10: (0, -INF), 200: (5, INF), 201: (D - 1, -INF), 350: (2, INF), 399: (7, -INF)}
    for key, (channel, x) in bad.items():
        b.k[0][key, 0, channel] = x * sign
    b.k[0][300, 0, 0] = b.k[0][300, 0, 7] = -INF * sign      # twice in one key
    b.write(0, 0, b.k[0], b.v[0])
    g = torch.Generator().manual_seed(45)
    q = torch.randn(n, H, D, generator=g)
    for channel, x in list(bad.values()) + [(0, -INF), (7, -INF)]:
        q[:, :, channel] = q[:, :, channel].abs().clamp(min=1e-6) * (1.0 if x < 0 else -1.0)
    q[::3, :, 0] = 1.0                       # exact in one part: the others are 0
    q[1::3, :, 0] = 0.333251953125           # 11 bits, and a rest
    q[:, 3, 0] *= -1.0                       # this head's score of key 10 is +inf
    q = q.to(M.DTYPES[io])
    left = torch.ones(L, dtype=torch.bool)
    left[list(bad) + [300]] = False
    k = b.k[0].clone()
    k[~left] = 0.0
    seen = M.visible(torch.arange(L - n, L), L, 0, 0) & left
    weight = 0.0 if io == "f32" else {"bf16": 2.0 ** -8, "f16": 2.0 ** -10}[io]
    want, tol = M.attention(q, k, b.v[0], seen, scale, M.io_eps(io), weight)
    want[:, 3] = NAN
    out = _prefill(b, H, q.view(n, -1).to(DEV), [n], scale)
    M.check(out, want, tol, "prompt")
    out = _decode(b, H, q[-1:].reshape(1, -1).to(DEV), scale)
    M.check(out, want[-1:], tol[-1:], "decode")


@pytest.mark.parametrize("dtype,io", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("H,Hkv,D,window,sinks", [(4, 1, 64, 0, 0), (17, 1, 100, 0, 0), (8, 2, 128, 0, 0), (4, 1, 256, 4500, 300), (6, 2, 36, 4500, 300)])
def test_decode_infinite_keys_among_many(H, Hkv, D, window, sinks, dtype, io):
    """Long rows in shares, of which one holds the infinite key; pages that are missing; an infinite value besides; and a row
    with a key that is no number beside one without."""
    _announce("infinite keys of long rows", H, Hkv, D, window, dtype, io)
    b = M.Batch([9001, 9001, 40], Hkv, D, 32, dtype, seed=D + 3)
    for s in (0, 1):
        b.k[s][6000, Hkv - 1, D - 1] = -INF
        b.k[s][100, 0, 2] = -INF
        b.v[s][6001, Hkv - 1, 3] = INF
        b.v[s][6000, 0, 3] = -1.5
        b.table[s, 200] = -1                 # positions 6400 to 6431
    b.k[1][8000, 0, 1] = NAN
    for s in range(3):
        for lo, hi in ((0, min(6400, b.lens[s])), (6432, b.lens[s])):
            if hi > lo:
                b.write(s, lo, b.k[s][lo:hi], b.v[s][lo:hi])
    q = torch.randn(3, H, D, generator=torch.Generator().manual_seed(46))
    q[:, :, D - 1], q[:, :, 2] = q[:, :, D - 1].abs() + 0.01, q[:, :, 2].abs() + 0.01
    q = q.to(M.DTYPES[io])
    out = _decode(b, H, q.view(3, -1).to(DEV), 0.1, window, sinks)
    for s in range(3):
        n = b.lens[s]
        there = (b.table[s].repeat_interleave(32)[:n] >= 0)[None]
        seen = M.visible(torch.tensor([n - 1]), n, window, sinks) & there
        for h in range(Hkv):
            heads = slice(h * (H // Hkv), (h + 1) * (H // Hkv))
            k, left = b.k[s][:, h:h + 1].clone(), seen.clone()
            gone = ~torch.isfinite(k).all(2)[:, 0]
            if bool((torch.isnan(k).any(2)[:, 0] & seen[0]).any()):
                assert bool(torch.isnan(out[s, heads]).all()), f"sequence {s}, kv head {h}: a key that is no number"
                continue
            left[0, gone] = False
            k[gone] = 0.0
            want, tol = M.attention(q[s:s + 1, heads], k, b.v[s][:, h:h + 1], left, 0.1, M.io_eps(io), 2.0 ** -15 if io != "f32" else 0.0)
            M.check(out[s:s + 1, heads], want, tol, f"sequence {s}, kv head {h}")
