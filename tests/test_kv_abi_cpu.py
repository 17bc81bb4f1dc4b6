"""Host-side checks of the cache's and the attention's entry points: sizes of pages and workspaces, and the status of every
refusal, before anything touches a GPU.  The binding's own refusals are those of its tensors."""
import ctypes

import pytest
import torch

import paper_2502_11880_amd as B

FAKE = 1 << 20          # aligned, never dereferenced: validation fails before any launch

pytestmark = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="placeholder device pointers: validation checks run without a GPU")

OK, INVALID, SHAPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 5


def _cache(**kw):
    a = dict(k=FAKE, v=FAKE, table=FAKE, kv_len=FAKE, n_pages=100, n_seqs=3, max_pages=20, page_size=32, n_kv_heads=8, head_dim=128,
             dtype=1)
    a.update(kw)
    return B._KvCache(*a.values())


def _pool(**kw):
    a = dict(k=FAKE, v=FAKE, n_layers=2, n_pages=100, k_page_bytes=4096, v_page_bytes=4096)
    a.update(kw)
    return B._KvPool(*a.values())


def _tables(**kw):
    a = dict(table=FAKE, kv_len=FAKE, refs=FAKE, n_seqs=3, max_pages=20, n_pages=100)
    a.update(kw)
    return B._KvTables(*a.values())


def _ref(s):
    return None if s is None else ctypes.byref(s)


def test_page_bytes():
    f = B.bitnet_kv_page_bytes
    assert f(1, 32, 8, 128, False) == f(2, 32, 8, 128, True) == 8 * 32 * 128 * 2
    assert f(2, 64, 3, 100, False) == 3 * 64 * 104 * 2 and f(2, 64, 3, 100, True) == 3 * 64 * 100 * 2
    for bad in ((0, 32, 8, 128), (3, 32, 8, 128), (1, 8, 8, 128), (1, 48, 8, 128), (1, 512, 8, 128), (1, 32, 0, 128), (1, 32, 1025, 128),
                (1, 32, 8, 0), (1, 32, 8, 102), (1, 32, 8, 260)):
        assert f(*bad, False) == 0


def test_workspace_bytes():
    f = B.bitnet_attn_decode_workspace_bytes
    assert f(1, 32, 8, 128, 16, 4) == 0                        # rows of 64 keys are never split
    assert f(1, 32, 8, 128, 16, 4096, 64, 4) == 0              # nor those of a short window, however long the cache
    assert f(1, 32, 8, 128, 16, 4096) > 0 and f(5, 32, 8, 128, 16, 4096) == f(1, 32, 8, 128, 16, 4096)
    for bad in ((1, 33, 8, 128, 16, 4096), (1, 32, 8, 130, 16, 4096), (1, 32, 8, 128, 24, 4096), (1, 0, 8, 128, 16, 4096),
                (1, 2048, 8, 128, 16, 4096), (1, 32, 8, 128, 16, 0), (1, 32, 8, 128, 16, 1 << 21), (1, 32, 8, 128, 16, 4096, -1, 0)):
        assert f(*bad) == 0
    g = B.bitnet_attn_prefill_workspace_bytes
    assert g(1, 1, 1, 64, 32, 8, 128, 64, 130) > 0             # few queries, many keys: split
    assert g(1, 1, 1, 64, 32, 8, 128, 64, 2) == 0              # few keys
    assert g(1, 1, 1, 4096, 32, 8, 128, 64, 130) == 0          # queries enough
    assert g(1, 0, 2, 64, 32, 8, 128, 64, 130, 64, 4) == 0     # a short window
    for bad in ((0, 0, 1, 64, 32, 8, 128, 64, 130), (1, 2, 1, 64, 32, 8, 128, 64, 130), (1, 1, 0, 64, 32, 8, 128, 64, 130),
                (1, 1, 1, 0, 32, 8, 128, 64, 130), (1, 1, 1, 64, 31, 8, 128, 64, 130), (1, 1, 1, 64, 32, 8, 126, 64, 130),
                (1, 1, 1, 64, 32, 8, 128, 60, 130), (1, 1, 1, 64, 32, 8, 128, 64, 0), (1, 1, 1, 64, 32, 8, 128, 64, 130, -1, 0)):
        assert g(*bad) == 0
    assert B.bitnet_kv_workspace_bytes(0, 1) == 0 and B.bitnet_kv_workspace_bytes(100, -1) == 0
    assert B.bitnet_kv_workspace_bytes(100, 0) >= 1200 and B.bitnet_kv_workspace_bytes(1 << 20, 64) >= 12 << 20


CACHE_FAULTS = [(None, INVALID), (dict(dtype=0), INVALID), (dict(dtype=7), INVALID), (dict(page_size=24), SHAPE), (dict(page_size=0), SHAPE),
                (dict(n_kv_heads=0), SHAPE), (dict(head_dim=126), SHAPE), (dict(head_dim=512), SHAPE), (dict(n_pages=0), SHAPE),
                (dict(n_pages=1 << 30), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(n_seqs=(1 << 20) + 1), SHAPE), (dict(max_pages=0), SHAPE),
                (dict(max_pages=(1 << 19) + 1), SHAPE), (dict(k=None), INVALID), (dict(table=None), INVALID), (dict(kv_len=None), INVALID),
                (dict(v=FAKE + 8), ALIGN), (dict(table=FAKE + 2), ALIGN)]


def _append(cache, k=FAKE, v=FAKE, src=0, start=FAKE, n=3):
    return B.lib().bitnet_kv_append(_ref(cache), k, v, src, start, n, None)


def _decode(cache, q=FAKE, dtype=0, heads=32, window=0, sinks=0, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return B.lib().bitnet_attn_decode(_ref(cache), q, dtype, heads, 1.0, window, sinks, out, ws, ws_bytes, None)


def _prefill(cache, q=FAKE, dtype=0, heads=32, start=FAKE, n=3, window=0, sinks=0, out=FAKE, ws=None):
    return B.lib().bitnet_attn_prefill(_ref(cache), q, dtype, heads, start, n, 1.0, window, sinks, out, ws, 0, None)


@pytest.mark.parametrize("fault,status", CACHE_FAULTS)
@pytest.mark.parametrize("call", [_append, _decode, _prefill])
def test_cache_refusals(call, fault, status):
    assert call(None if fault is None else _cache(**fault)) == status
    assert B.bitnet_last_error()


def test_append_refusals():
    c = _cache()
    assert _append(c, k=None) == INVALID and _append(c, v=None) == INVALID
    assert _append(c, k=FAKE + 4) == ALIGN and _append(c, start=FAKE + 1) == ALIGN
    assert _append(c, src=2) == INVALID and _append(c, src=9) == INVALID
    assert _append(c, n=-1) == SHAPE and _append(c, n=(1 << 24) + 1) == SHAPE
    assert _append(c, start=None, n=4) == SHAPE                # one token each: as many as sequences
    assert _append(c, k=None, v=None, n=0) == OK and _append(_cache(n_seqs=0, k=None, table=None), n=0) == OK


def test_attention_refusals():
    c = _cache()
    for call in (_decode, _prefill):
        assert call(c, q=None) == INVALID and call(c, out=None) == INVALID
        assert call(c, q=FAKE + 8) == ALIGN and call(c, out=FAKE + 4) == ALIGN
        assert call(c, dtype=2) == INVALID and call(c, dtype=-1) == INVALID
        assert call(c, heads=0) == SHAPE and call(c, heads=33) == SHAPE and call(c, heads=2048) == SHAPE
        assert call(c, window=-1) == INVALID and call(c, sinks=-1) == INVALID
    need = B.bitnet_attn_decode_workspace_bytes(3, 32, 8, 128, 32, 20)
    assert need > 0
    assert _decode(c, ws=None) == WORKSPACE and _decode(c, ws_bytes=need - 1) == WORKSPACE and _decode(c, ws=FAKE + 4) == ALIGN
    assert "workspace" not in B.bitnet_status_string(OK)
    assert _decode(_cache(n_seqs=0, k=None), q=None, out=None, ws=None, ws_bytes=0) == OK
    assert _prefill(c, start=None) == INVALID and _prefill(c, start=FAKE + 2) == ALIGN
    assert _prefill(c, n=-1) == SHAPE and _prefill(c, n=(1 << 24) + 1) == SHAPE and _prefill(c, heads=1024, n=(1 << 20) + 1) == SHAPE
    assert _prefill(_cache(n_seqs=1 << 20), n=3) == SHAPE
    assert _prefill(c, n=0, q=None, out=None) == OK
    assert _prefill(c, ws=FAKE + 4) == ALIGN


def test_page_call_refusals():
    lib = B.lib()
    need = B.bitnet_kv_workspace_bytes(100, 3)

    def reserve(t=None, seqs=FAKE, n_new=FAKE, n=2, page=16, short=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return lib.bitnet_kv_reserve(_ref(t or _tables()), seqs, n_new, n, page, short, ws, ws_bytes, None)

    def fork(p=None, t=None, parents=FAKE, children=FAKE, n=2, page=16, short=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return lib.bitnet_kv_fork(_ref(p or _pool()), _ref(t or _tables()), parents, children, n, page, short, ws, ws_bytes, None)

    def compact(p=None, t=None, live=FAKE, ws=FAKE, ws_bytes=1 << 30):
        return lib.bitnet_kv_compact(_ref(p or _pool()), _ref(t or _tables()), live, ws, ws_bytes, None)

    def free(t=None, seqs=FAKE, n=2):
        return lib.bitnet_kv_free(_ref(t or _tables()), seqs, n, None)

    def trim(t=None, seqs=FAKE, n=2, page=16, window=8, sinks=4):
        return lib.bitnet_kv_trim(_ref(t or _tables()), seqs, n, page, window, sinks, None)

    for bad, status in ((dict(refs=None), INVALID), (dict(refs=FAKE + 2), ALIGN), (dict(table=None), INVALID), (dict(table=FAKE + 1), ALIGN),
                        (dict(n_pages=0), SHAPE), (dict(n_seqs=-1), SHAPE), (dict(max_pages=0), SHAPE), (dict(max_pages=1 << 21), SHAPE)):
        for call in (reserve, fork, compact, free, trim):
            # a pool that does not go with the tables is another fault
            if call in (fork, compact) and "n_pages" in bad:
                continue
            assert call(t=_tables(**bad)) == status, (call.__name__, bad)
    for call in (reserve, fork, free, trim):
        assert call(t=_tables(kv_len=None)) == INVALID
        assert call(n=4) == SHAPE and call(n=-1) == SHAPE
    for call in (reserve, fork, trim):
        assert call(page=20) == SHAPE
    for call in (reserve, fork, compact):
        assert call(ws=None) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE and call(ws=FAKE + 8) == ALIGN
    assert reserve(seqs=None) == INVALID and reserve(n_new=None) == INVALID and reserve(short=None) == INVALID
    assert reserve(seqs=FAKE + 2) == ALIGN
    assert fork(parents=None) == INVALID and fork(children=FAKE + 2) == ALIGN and fork(short=None) == INVALID
    assert free(seqs=None) == INVALID and trim(seqs=None) == INVALID and free(n=0, seqs=None) == OK and trim(n=0, seqs=None) == OK
    assert trim(window=0) == INVALID and trim(sinks=-1) == INVALID
    assert compact(live=None) == INVALID and compact(p=_pool(n_pages=99)) == SHAPE and fork(p=_pool(n_pages=99)) == SHAPE

    for bad, status in ((dict(k=None), INVALID), (dict(v=FAKE + 8), ALIGN), (dict(n_layers=0), SHAPE), (dict(n_layers=70000), SHAPE),
                        (dict(k_page_bytes=100), SHAPE), (dict(v_page_bytes=0), SHAPE), (dict(k_page_bytes=(1 << 30) + 16), SHAPE)):
        assert fork(p=_pool(**bad)) == status and compact(p=_pool(**bad)) == status
        assert lib.bitnet_kv_copy_pages(_ref(_pool(**bad)), FAKE, FAKE, 1, None) == status
    copy = lib.bitnet_kv_copy_pages
    assert copy(_ref(_pool()), None, FAKE, 1, None) == INVALID and copy(_ref(_pool()), FAKE, FAKE + 1, 1, None) == ALIGN
    assert copy(_ref(_pool()), FAKE, FAKE, -1, None) == SHAPE and copy(_ref(_pool()), None, None, 0, None) == OK


def test_binding_refuses_tensors_that_do_not_fit():
    k, v = torch.zeros(4, 2, 13, 32, 8, dtype=torch.float16), torch.zeros(4, 2, 4, 100, 8, dtype=torch.float16)
    table, lens = torch.zeros(3, 5, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for bad in ((k[:, :, :12], v), (k, v[:3]), (k[0], v), (k, v[:, :, :2])):
        with pytest.raises(ValueError):
            B._cache(*bad, table, lens)
    with pytest.raises(TypeError):
        B._cache(k, v.to(torch.bfloat16), table, lens)
    with pytest.raises(ValueError):
        B._cache(k, v, table, lens[:2])
    with pytest.raises(TypeError):                             # a host tensor
        B._cache(k, v, table, lens)
    with pytest.raises(ValueError):
        B._pool(k[None], v[None, :3])
    with pytest.raises(ValueError):
        B._rows(torch.zeros(3, 199), "k", 200)
