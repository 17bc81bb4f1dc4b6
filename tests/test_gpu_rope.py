"""The position rotation against its definition in 64 bits, and the append that rotates against the two calls it joins."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import hip_runner as H
from tests import kv_model as M

pytestmark = pytest.mark.gpu
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}       # of the last rounding; that of 32 bits is counted below
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}


def _freqs(rot, theta=10000.0):
    return torch.tensor([theta ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)], dtype=torch.float64)


def _turned(x, pos, freqs, interleaved, gain):
    """(out, tolerance) of x [n, heads, dim] in 64 bits.  cos and sin carry half a step of 32 bits each, a product and the sum
    another, and the angle 2^-53 of its turns, which at 2^31 positions of up to 1 / 2 pi turns is 2^-22 of a radian."""
    rot = 2 * freqs.numel()
    x = x.double()
    t = pos.double()[:, None] * freqs
    t = (t - t.round()) * (2 * math.pi)
    c, s = (gain * t.cos())[:, None], (gain * t.sin())[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out, tol = x.clone(), torch.zeros_like(x)
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    u = 2.0 ** -24
    angle = (2.0 ** -52 * 2 * math.pi * pos.double().abs()[:, None] * freqs)[:, None] * abs(gain)
    size = x[..., a].abs() + x[..., b].abs()
    tol[..., a] = 2 * u * ((x[..., a] * c).abs() + (x[..., b] * s).abs()) + u * out[..., a].abs() + angle * size
    tol[..., b] = 2 * u * ((x[..., b] * c).abs() + (x[..., a] * s).abs()) + u * out[..., b].abs() + angle * size
    return out, tol


def _check(got, want, tol, io, what):
    err = (got.double().cpu() - want).abs()
    assert bool((err <= tol * (1 + HALF_STEP[io]) + HALF_STEP[io] * want.abs() + TINY[io]).all()), f"{what}: worst {float(err.max())}"


SHAPES = [(1, 1, 4, 2), (1, 32, 128, 128), (7, 8, 128, 64), (3, 5, 100, 74), (2, 3, 100, 100), (5, 1, 256, 256), (4, 7, 64, 62), (2, 2, 256, 2),
          (300, 4, 96, 96), (2100, 2, 80, 40), (3, 1024, 8, 8), (9, 64, 12, 6)]


@pytest.mark.parametrize("io", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,dim,rot", SHAPES)
def test_rope(n, heads, dim, rot, interleaved, io):
    print("case: rope", n, heads, dim, rot, interleaved, io, flush=True)
    g = torch.Generator().manual_seed(n + heads + dim + rot)
    x = torch.randn(n, heads, dim, generator=g).to(T[io])
    pos = torch.randint(0, 1 << 24, (n,), generator=g).to(torch.int32)
    pos[0] = 0 if n > 1 else 5
    gain = 1.0 if n % 2 else 1.2
    f = _freqs(rot)
    want, tol = _turned(x, pos, f, interleaved, torch.tensor(gain).double().item())
    dev = x.view(n, -1).to(H.DEV)
    out = torch.full_like(dev, float("nan"))
    B.bitnet_rope(dev, pos.to(H.DEV), f.to(H.DEV), out, dim, interleaved, gain)
    _check(out.view(n, heads, dim), want, tol + 2.0 ** -24 * want.abs() * (gain != 1.0), io, "rope")
    assert torch.equal(dev.cpu(), x.view(n, -1))
    B.bitnet_rope(dev, pos.to(H.DEV), f.to(H.DEV), dev, dim, interleaved, gain)       # in place
    assert torch.equal(dev, out)


def test_far_and_negative_positions():
    pos = torch.tensor([0, 1, -1, 12345, -12345, (1 << 24) - 1, 1 << 24, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    x = torch.randn(len(pos), 2, 128, generator=torch.Generator().manual_seed(3))
    f = _freqs(128, 500000.0)
    want, tol = _turned(x, pos, f, False, 1.0)
    out = torch.empty(len(pos), 256, device=H.DEV)
    B.bitnet_rope(x.view(-1, 256).to(H.DEV), pos.to(H.DEV), f.to(H.DEV), out, 128)
    _check(out.view(x.shape), want, tol, "f32", "far")
    assert torch.equal(out[0].cpu(), x[0].view(-1))                                    # position 0 turns nothing


def test_turning_back_is_the_inverse():
    """Opposite positions undo each other to the roundings of both."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(40, 3, 64, generator=g)
    pos = torch.randint(0, 1 << 20, (40,), generator=g).to(torch.int32)
    f = _freqs(64).to(H.DEV)
    a, b = torch.empty(40, 192, device=H.DEV), torch.empty(40, 192, device=H.DEV)
    B.bitnet_rope(x.view(40, -1).to(H.DEV), pos.to(H.DEV), f, a, 64)
    B.bitnet_rope(a, (-pos).to(H.DEV), f, b, 64)
    size = x.abs() + torch.cat([x[..., 32:], x[..., :32]], -1).abs()
    assert bool(((b.view(x.shape).cpu() - x).abs() <= 12 * 2.0 ** -24 * size).all())


def test_rope_past_two_to_the_31st_value():
    n, heads, dim = 262300, 64, 128
    print("case: rope of 2^31 values and more", flush=True)
    x = torch.zeros(n, heads * dim, dtype=torch.float16, device=H.DEV)
    g = torch.Generator().manual_seed(5)
    last = torch.randn(2, heads, dim, generator=g).half()
    x[-2:] = last.view(2, -1).to(H.DEV)
    pos = torch.arange(n, dtype=torch.int32, device=H.DEV)
    f = _freqs(dim)
    B.bitnet_rope(x, pos, f.to(H.DEV), x, dim)
    want, tol = _turned(last, torch.tensor([n - 2, n - 1]), f, False, 1.0)
    _check(x[-2:].view(2, heads, dim), want, tol, "f16", "last rows")
    assert not bool(x[:4096].any())


def _scaled(rot, theta, kind, factor, original, low, high):
    out = []
    base = theta * factor ** (rot / (rot - 2)) if kind == "base" else theta
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot) / (2 * math.pi)
        w = 1.0
        if kind == "linear":
            w = 0.0
        elif kind == "turns":
            w = min(1.0, max(0.0, (original * f - low) / (high - low)))
        elif kind == "index":
            lo = max(0, math.floor(rot * math.log(original / (high * 2 * math.pi)) / (2 * math.log(theta))))
            hi = min(rot - 1, math.ceil(rot * math.log(original / (low * 2 * math.pi)) / (2 * math.log(theta))))
            w = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
        out.append(f * w + f / factor * (1 - w))
    return torch.tensor(out, dtype=torch.float64)


@pytest.mark.parametrize("kind", ["none", "linear", "base", "turns", "index"])
@pytest.mark.parametrize("rot,theta,factor,original,low,high", [(128, 10000.0, 8.0, 4096, 1.0, 32.0), (4, 500000.0, 2.5, 8192, 1.0, 4.0),
                                                                (256, 1e6, 40.0, 100, 0.5, 7.0), (74, 10000.0, 0.5, 30000, 1.0, 4.0)])
def test_frequencies(kind, rot, theta, factor, original, low, high):
    """A power is good to an ulp or two, its exponent to half an ulp times a logarithm of up to 14 + 3.7 of its size."""
    want = _scaled(rot, theta, kind, factor, original, low, high)
    got = torch.full((rot // 2,), float("nan"), dtype=torch.float64, device=H.DEV)
    B.bitnet_rope_freqs(got, theta, kind, factor, original, low, high)
    # the ramp of `turns` divides by (high - low) >= 3: its own error is a few ulps of original f / 3 <= high
    assert bool(((got.cpu() - want).abs() <= 64 * 2.0 ** -53 * want * (1 + original / 3 * (kind == "turns"))).all())
    assert bool((got > 0).all()) and (factor < 1 or bool((got[1:] < got[:-1]).all()))


def test_frequencies_of_one_pair():
    got = torch.zeros(1, dtype=torch.float64, device=H.DEV)
    B.bitnet_rope_freqs(got, 10000.0)
    assert abs(got.item() * 2 * math.pi - 1) < 1e-15


# ---------------------------------------------------------------------------------------------------------------------
# Appending
# ---------------------------------------------------------------------------------------------------------------------
def _append_both(b, new, heads, rot, interleaved, io, seed, gain=1.0, with_q=True, start=None):
    """The joined call, and bitnet_rope then bitnet_kv_append, on the same inputs: (caches, q) of either."""
    g = torch.Generator().manual_seed(seed)
    n = sum(new) if start is None else start[-1]
    dim, hk = b.dim, b.heads
    q, k, v = (torch.randn(n, h * dim, generator=g).to(T[io]).to(H.DEV) for h in (heads, hk, hk))
    starts = [sum(new[:i]) for i in range(len(new) + 1)] if start is None else start
    start = torch.tensor(starts, dtype=torch.int32, device=H.DEV)
    f = _freqs(rot).to(H.DEV)
    kc, vc, table, kv_len = b.on(H.DEV)
    kc2, vc2 = kc.clone(), vc.clone()
    q_out = torch.full_like(q, 77.0) if with_q else None
    B.bitnet_kv_append_rope(k, v, start, kc, vc, table, kv_len, f, interleaved, gain, q if with_q else None, q_out)
    pos = torch.zeros(n, dtype=torch.int32)
    owned = torch.zeros(n, dtype=torch.bool)
    for s, total in enumerate(b.kv_len.tolist()):
        first, count = starts[s], starts[s + 1] - starts[s]
        for i in range(count):
            pos[first + i] = total - count + i
            owned[first + i] = total - count + i >= 0
    pos = pos.to(H.DEV)
    kr, qr = torch.empty_like(k), torch.empty_like(q)
    B.bitnet_rope(k, pos, f, kr, dim, interleaved, gain)
    B.bitnet_rope(q, pos, f, qr, dim, interleaved, gain)
    B.bitnet_kv_append(kr, v, start, kc2, vc2, table, kv_len)
    qr[~owned.to(H.DEV)] = 77.0
    return (kc, vc, q_out), (kc2, vc2, qr)


def _same(a, b, what):
    assert torch.equal(torch.nan_to_num(a.float(), 12345.0), torch.nan_to_num(b.float(), 12345.0)), what


@pytest.mark.parametrize("cache,io", [("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("heads,kv_heads,dim,rot,interleaved", [(8, 2, 128, 128, False), (4, 4, 100, 64, True), (6, 3, 100, 74, False),
                                                                (16, 1, 64, 32, True), (5, 5, 36, 34, True), (2, 1, 256, 256, False)])
@pytest.mark.parametrize("page,new,past", [(16, [1, 1, 1], [0, 15, 37]), (32, [37, 0, 1, 64, 5], [0, 9, 31, 0, 250]), (128, [300], [77])])
def test_append_is_rope_then_append(cache, io, heads, kv_heads, dim, rot, interleaved, page, new, past):
    print("case: append", cache, io, heads, kv_heads, dim, rot, interleaved, page, flush=True)
    b = M.Batch([a + p for a, p in zip(new, past)], kv_heads, dim, page, cache, seed=page + dim)
    got, want = _append_both(b, new, heads, rot, interleaved, io, 7, gain=1.1)
    for a, w, what in zip(got, want, ("keys", "values", "q")):
        _same(a, w, what)


def test_append_of_one_token_each():
    b = M.Batch([1, 16, 17, 40], 2, 128, 16, "bf16", seed=2)
    kc, vc, table, kv_len = b.on(H.DEV)
    k, v, q = (torch.randn(4, h * 128, device=H.DEV) for h in (2, 2, 8))
    f = _freqs(128).to(H.DEV)
    outs = []
    for start in (None, torch.arange(5, dtype=torch.int32, device=H.DEV)):
        kk, vv, qq = kc.clone(), vc.clone(), q.clone()
        B.bitnet_kv_append_rope(k, v, start, kk, vv, table, kv_len, f, q=qq, q_out=qq)
        outs.append((kk, vv, qq))
    for a, w in zip(*outs):
        _same(a, w, "with and without offsets")


def test_append_against_the_definition():
    """Keys as the cache holds them: the 64-bit rotation, rounded once."""
    for cache in ("bf16", "f16"):
        new, past = [5, 21], [3, 0]
        b = M.Batch([a + p for a, p in zip(new, past)], 2, 100, 16, cache, seed=3)
        g = torch.Generator().manual_seed(9)
        k, v = torch.randn(26, 2, 100, generator=g), torch.randn(26, 2, 100, generator=g)
        kc, vc, table, kv_len = b.on(H.DEV)
        start = torch.tensor([0, 5, 26], dtype=torch.int32, device=H.DEV)
        f = _freqs(48)
        B.bitnet_kv_append_rope(k.view(26, -1).to(H.DEV), v.view(26, -1).to(H.DEV), start, kc, vc, table, kv_len, f.to(H.DEV), True)
        pos = torch.cat([torch.arange(3, 8), torch.arange(0, 21)])
        want, tol = _turned(k, pos, f, True, 1.0)
        kc, vc = kc.cpu(), vc.cpu()
        for i in range(26):
            s = 0 if i < 5 else 1
            page, slot = int(b.table[s][int(pos[i]) // 16]), int(pos[i]) % 16
            got = kc[page, :, :, slot].reshape(2, -1)
            _check(got[:, :100], want[i], tol[i], cache, "keys")
            assert not bool(got[:, 100:].any())
            assert torch.equal(vc[page, :, slot // 8, :, slot % 8], v[i].to(T[cache]))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_append_where_tokens_have_no_place(io):
    """Missing pages, lengths that are too short or past the table, offsets that start past 0: the same as the two calls, and no
    row of q that no sequence owns."""
    b = M.Batch([40, 20, 9, 33], 2, 64, 16, "bf16", seed=4)
    b.table[0, 1] = -1
    b.table[3, 2] = b.pages + 5
    b.kv_len = torch.tensor([40, 3, 0, 200], dtype=torch.int32)       # 20 new tokens but a length of 3; none; past the table
    got, want = _append_both(b, [17, 20, 9, 30], 4, 64, False, io, 11)
    for a, w, what in zip(got, want, ("keys", "values", "q")):
        _same(a, w, what)
    # offsets from 5 on: the first rows belong to nobody
    b = M.Batch([10, 12], 2, 64, 16, "bf16", seed=5)
    got, want = _append_both(b, None, 4, 64, True, io, 12, start=[5, 15, 27])
    for a, w, what in zip(got, want, ("keys", "values", "q")):
        _same(a, w, what)
    assert bool((got[2][:5] == 77.0).all())


def test_append_without_q():
    b = M.Batch([10, 70], 3, 96, 64, "f16", seed=6)
    got, want = _append_both(b, [10, 33], 3, 96, False, "f32", 13, with_q=False)
    _same(got[0], want[0], "keys")
    _same(got[1], want[1], "values")


def test_binding_refusals():
    e = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device=H.DEV)  # noqa: E731
    i = lambda n: torch.zeros(n, dtype=torch.int32, device=H.DEV)  # noqa: E731
    f = e(32, t=torch.float64)
    B.bitnet_rope(e(0, 128), i(0), f, e(0, 128), 64)
    for args, err in (((e(2, 100), i(2), f, e(2, 100), 64), ValueError), ((e(2, 128), i(3), f, e(2, 128), 64), ValueError),
                      ((e(2, 128), i(2), f, e(2, 128, t=torch.float16), 64), ValueError), ((e(2, 128), i(2), f.float(), e(2, 128), 64), TypeError),
                      ((e(2, 128), i(2).long(), f, e(2, 128), 64), TypeError), ((e(2, 120), i(2), f, e(2, 120), 60), B.BitnetError)):
        with pytest.raises(err):
            B.bitnet_rope(*args)
    b = M.Batch([4, 4], 2, 64, 16, "bf16", seed=1)
    kc, vc, table, kv_len = b.on(H.DEV)
    for kw, err in ((dict(q=e(2, 256)), ValueError), (dict(q=e(2, 256), q_out=e(2, 128)), ValueError), (dict(q=e(3, 256), q_out=e(3, 256)), ValueError),
                    (dict(q=e(2, 192), q_out=e(2, 192)), B.BitnetError), (dict(q=e(2, 256, t=torch.bfloat16), q_out=e(2, 256, t=torch.bfloat16)), ValueError)):
        with pytest.raises(err):
            B.bitnet_kv_append_rope(e(2, 128), e(2, 128), None, kc, vc, table, kv_len, f, **kw)
