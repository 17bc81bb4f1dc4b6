"""Refusals of the norm, the rotation and the append that rotates: the documented status before anything touches a GPU."""
import ctypes

import pytest

import paper_2502_11880_amd as B
from tests.test_abi_cpu import FAKE, cpu_only

BIG = 1 << 40                # places of distinct buffers that never overlap


def _norm(**kw):
    a = dict(x=FAKE, xd=0, res=BIG, out=2 * BIG, rd=0, gamma=3 * BIG, eps=1e-5, M=4, K=64, y=4 * BIG, yd=0, xq=5 * BIG, s=6 * BIG, rs=7 * BIG)
    a.update(kw)
    return B.lib().bitnet_norm_quantize(a["x"], a["xd"], a["res"], a["out"], a["rd"], a["gamma"], a["eps"], a["M"], a["K"], a["y"],
                                        a["yd"], a["xq"], a["s"], a["rs"], None)


@cpu_only
@pytest.mark.parametrize("status,kw", [
    (1, dict(x=None)), (1, dict(xd=3)), (1, dict(rd=-1)), (1, dict(yd=7)), (1, dict(xd=1, rd=0)), (1, dict(xd=1, rd=2)),
    (1, dict(res=None)), (1, dict(y=None, xq=None, s=None, rs=None)), (1, dict(s=None)), (1, dict(xq=None)), (1, dict(xq=None, s=None)),
    (1, dict(eps=0.0)), (1, dict(eps=-1.0)), (1, dict(eps=float("nan"))), (1, dict(eps=float("inf"))),
    (2, dict(M=-1)), (2, dict(M=(1 << 24) + 1)), (2, dict(K=0)), (2, dict(K=1048577)),
    (3, dict(x=FAKE + 4)), (3, dict(res=BIG + 8)), (3, dict(out=2 * BIG + 2)), (3, dict(gamma=3 * BIG + 4)), (3, dict(y=4 * BIG + 8)),
    (3, dict(xq=5 * BIG + 1)), (3, dict(s=6 * BIG + 2)), (3, dict(rs=7 * BIG + 1)),
    # overlaps: outputs with one another, with an input that has another type, or one that starts elsewhere
    (1, dict(y=2 * BIG)), (1, dict(xq=2 * BIG)), (1, dict(rs=6 * BIG + 4)), (1, dict(y=FAKE, yd=1)), (1, dict(out=FAKE + 16)),
    (1, dict(xq=FAKE)), (1, dict(s=BIG)), (1, dict(y=3 * BIG)), (1, dict(out=BIG, rd=1, y=BIG, yd=1))])
def test_norm_refusals(status, kw):
    assert _norm(**kw) == status, B.bitnet_last_error()


@cpu_only
def test_norm_of_no_rows():
    assert _norm(M=0) == 0 and _norm(M=0, x=None, res=None, out=None) == 0


@cpu_only
@pytest.mark.parametrize("status,kw", [
    (1, dict(kind=5)), (1, dict(kind=-1)), (2, dict(rot=0)), (2, dict(rot=7)), (2, dict(rot=258)), (1, dict(theta=1.0)),
    (1, dict(theta=float("inf"))), (1, dict(theta=float("nan"))), (1, dict(kind=1, factor=0.0)), (1, dict(kind=2, factor=float("nan"))),
    (2, dict(kind=2, rot=2)), (1, dict(kind=3, original=0.0)), (1, dict(kind=3, low=0.0)), (1, dict(kind=4, low=4.0, high=4.0)),
    (1, dict(kind=4, high=float("inf"))), (1, dict(freqs=None)), (3, dict(freqs=FAKE + 4))])
def test_freqs_refusals(status, kw):
    a = dict(kind=0, theta=10000.0, rot=64, factor=2.0, original=4096.0, low=1.0, high=4.0, freqs=FAKE)
    a.update(kw)
    got = B.lib().bitnet_rope_freqs(a["kind"], a["theta"], a["rot"], a["factor"], a["original"], a["low"], a["high"], a["freqs"], None)
    assert got == status, B.bitnet_last_error()


def _rot(freqs=FAKE, rot=64, interleaved=0, gain=1.0):
    return B._Rotation(freqs, rot, interleaved, gain)


ROTATIONS = [(1, dict(freqs=None)), (3, dict(freqs=FAKE + 4)), (2, dict(rot=0)), (2, dict(rot=63)), (2, dict(rot=130)),
             (1, dict(interleaved=2)), (1, dict(interleaved=-1))]


@cpu_only
@pytest.mark.parametrize("status,rot,kw", [(s, r, {}) for s, r in ROTATIONS] + [(s, {}, k) for s, k in [
    (1, dict(x=None)), (1, dict(pos=None)), (1, dict(out=None)), (1, dict(dtype=3)), (2, dict(n=-1)), (2, dict(n=(1 << 24) + 1)),
    (2, dict(heads=0)), (2, dict(heads=1025)), (2, dict(dim=126)), (2, dict(dim=260)), (2, dict(dim=0)), (3, dict(x=FAKE + 8)),
    (3, dict(out=BIG + 4)), (3, dict(pos=2 * BIG + 2)), (1, dict(out=FAKE + 16)), (1, dict(x=FAKE + 4 * 3 * 128 * 4, out=FAKE + 16))]])
def test_rope_refusals(status, rot, kw):
    a = dict(x=FAKE, dtype=0, n=3, heads=4, dim=128, pos=2 * BIG, out=BIG)
    a.update(kw)
    got = B.lib().bitnet_rope(ctypes.byref(_rot(**rot)), a["x"], a["dtype"], a["n"], a["heads"], a["dim"], a["pos"], a["out"], None)
    assert got == status, B.bitnet_last_error()
    assert B.lib().bitnet_rope(None, FAKE, 0, 3, 4, 128, FAKE, FAKE, None) == 1
    assert B.lib().bitnet_rope(ctypes.byref(_rot()), None, 0, 0, 4, 128, None, None, None) == 0       # no tokens


def _cache(**kw):
    a = dict(k=FAKE, v=2 * FAKE, table=3 * FAKE, kv_len=4 * FAKE, n_pages=4, n_seqs=2, max_pages=2, ps=16, heads=2, dim=128, dtype=1)
    a.update(kw)
    return B._KvCache(a["k"], a["v"], a["table"], a["kv_len"], a["n_pages"], a["n_seqs"], a["max_pages"], a["ps"], a["heads"], a["dim"], a["dtype"])


@cpu_only
@pytest.mark.parametrize("status,rot,cache,kw", [(s, r, {}, {}) for s, r in ROTATIONS] + [
    (1, {}, dict(dtype=0), {}), (2, {}, dict(ps=24), {}), (2, {}, dict(dim=130), {}), (1, {}, dict(k=None), {}), (3, {}, dict(v=FAKE + 8), {}),
    (1, {}, {}, dict(src=2)), (2, {}, {}, dict(n=-1)), (2, {}, {}, dict(start=None, n=3)), (1, {}, {}, dict(k=None)), (1, {}, {}, dict(v=None)),
    (1, {}, {}, dict(q=None)), (1, {}, {}, dict(q_out=None)), (2, {}, {}, dict(heads=3)), (2, {}, {}, dict(heads=0)), (2, {}, {}, dict(heads=1026)),
    (3, {}, {}, dict(q=BIG + 4)), (3, {}, {}, dict(q_out=2 * BIG + 8)), (3, {}, {}, dict(k=3 * BIG + 2)), (3, {}, {}, dict(start=5 * BIG + 1)),
    (1, {}, {}, dict(q_out=BIG + 16)), (1, {}, {}, dict(q_out=3 * BIG)), (1, {}, {}, dict(q_out=4 * BIG - 16))])
def test_append_rope_refusals(status, rot, cache, kw):
    a = dict(q=BIG, heads=4, k=3 * BIG, v=4 * BIG, src=0, start=5 * BIG, n=5, q_out=2 * BIG)
    a.update(kw)
    c, r = _cache(**cache), _rot(**rot)
    call = lambda: B.lib().bitnet_kv_append_rope(ctypes.byref(c), ctypes.byref(r), a["q"], a["heads"], a["k"], a["v"], a["src"],  # noqa: E731
                                                 a["start"], a["n"], a["q_out"], None)
    assert call() == status, B.bitnet_last_error()
    assert B.lib().bitnet_kv_append_rope(None, ctypes.byref(r), None, 0, FAKE, FAKE, 0, FAKE, 5, None, None) == 1
    assert B.lib().bitnet_kv_append_rope(ctypes.byref(_cache()), None, None, 0, FAKE, FAKE, 0, FAKE, 5, None, None) == 1


@cpu_only
def test_nothing_to_append():
    assert B.lib().bitnet_kv_append_rope(ctypes.byref(_cache()), ctypes.byref(_rot()), None, 0, None, None, 0, None, 0, None, None) == 2
    assert B.lib().bitnet_kv_append_rope(ctypes.byref(_cache()), ctypes.byref(_rot()), None, 0, None, None, 0, FAKE, 0, None, None) == 0
    none = _cache(n_seqs=0)
    assert B.lib().bitnet_kv_append_rope(ctypes.byref(none), ctypes.byref(_rot()), None, 0, None, None, 0, None, 0, None, None) == 0


def _shared(cache=None, **kw):
    a = dict(q=FAKE, dtype=0, heads=4, start=FAKE, prefix=FAKE, groups=2, scale=1.0, window=0, sinks=0, out=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    c = _cache(**(cache or {}))
    return B.lib().bitnet_attn_decode_shared(ctypes.byref(c), a["q"], a["dtype"], a["heads"], a["start"], a["prefix"], a["groups"], a["scale"],
                                             a["window"], a["sinks"], a["out"], a["ws"], a["ws_bytes"], None)


@cpu_only
@pytest.mark.parametrize("status,cache,kw", [
    (1, dict(dtype=0), {}), (2, dict(ps=48), {}), (2, dict(dim=2), {}), (1, dict(table=None), {}), (3, dict(k=FAKE + 8), {}),
    (1, {}, dict(dtype=2)), (2, {}, dict(heads=3)), (2, {}, dict(heads=0)), (2, {}, dict(heads=1026)), (1, {}, dict(window=-1)), (1, {}, dict(sinks=-1)),
    (2, {}, dict(groups=3)), (2, {}, dict(groups=-1)), (1, {}, dict(q=None)), (1, {}, dict(out=None)), (1, {}, dict(start=None)),
    (1, {}, dict(prefix=None)), (3, {}, dict(q=FAKE + 4)), (3, {}, dict(start=FAKE + 2)), (3, {}, dict(prefix=FAKE + 1))])
def test_shared_refusals(status, cache, kw):
    assert _shared(cache, **kw) == status, B.bitnet_last_error()


@cpu_only
def test_shared_workspace_and_nothing_to_do():
    need = B.bitnet_attn_decode_shared_workspace_bytes(2, 4, 2, 128, 16, 2)
    if need:
        assert _shared(ws=None) == 5 and _shared(ws_bytes=need - 1) == 5 and _shared(ws=FAKE + 8, ws_bytes=need) == 3
    assert _shared(groups=0, q=None, out=None) == 0
    assert _shared(dict(n_seqs=0), groups=0) == 0
    sizes = [B.bitnet_attn_decode_shared_workspace_bytes(n, 32, 8, 128, 32, 100) for n in (1, 2, 16, 64, 1000, 1024, 5000)]
    assert sizes == sorted(sizes)                                    # it serves fewer sequences too
    assert B.bitnet_attn_decode_shared_workspace_bytes(4, 3, 2, 128, 32, 100) == 0
    assert B.bitnet_attn_decode_shared_workspace_bytes(4, 4, 2, 130, 32, 100) == 0
