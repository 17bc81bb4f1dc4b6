"""The workspace of a prompt call, on the CPU: bounded whatever the batch looks like, and independent of sequences that bring no
tokens."""
import pytest

import paper_2502_11880_amd as B

# as many rows of out as work groups fit the device have columns: 512 of 128 and 256 of 256, at up to 130 floats a row (heads of up
# to 128), or 256 of 128 at 258; an odd number of parts is held as one more
MOST = 65536 * 130 * 4 * 3 // 2
F32, BF16, F16 = 0, 1, 2


def _bytes(n_seqs, n_tokens, cache=BF16, io=BF16, heads=32, kv_heads=8, dim=128, page=64, max_pages=130, window=0, sinks=0):
    return B.bitnet_attn_prefill_workspace_bytes(cache, io, n_seqs, n_tokens, heads, kv_heads, dim, page, max_pages, window, sinks)


@pytest.mark.parametrize("cache,io", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("heads,kv_heads", [(32, 8), (32, 32), (1, 1), (3, 3), (40, 8), (16, 1), (1024, 1024), (1024, 1)])
@pytest.mark.parametrize("dim", [4, 64, 96, 100, 128, 192, 256])
def test_prefill_workspace_is_bounded(heads, kv_heads, dim, cache, io):
    for n_seqs in (1, 2, 12, 64, 256, 1000, 4096, 1 << 20):
        if n_seqs * kv_heads > 1 << 22:
            continue
        for n_tokens in (1, 2, 3, 17, 64, 200, 512, 1000, 4096, 30000):
            if n_tokens * heads > 1 << 30:
                continue
            for max_pages in (1, 16, 130, 4096, 1 << 18):
                assert _bytes(n_seqs, n_tokens, cache, io, heads, kv_heads, dim, max_pages=max_pages) <= MOST


def test_prefill_workspace_of_batches_with_many_sequences():
    assert _bytes(64, 64) <= MOST                              # a token each
    assert _bytes(256, 64) <= MOST and _bytes(4096, 64) <= MOST
    one = _bytes(1, 64)
    assert 0 < _bytes(64, 64) <= one and 0 < _bytes(256, 64) <= one
    # sequences past the tokens there are cannot have any
    assert _bytes(64, 64) == _bytes(256, 64) == _bytes(1024, 64)
    # a chunk is split beside 31 rows without tokens as well, also where many tokens would take the larger work groups
    assert _bytes(32, 64, F16, F32) > 0 and _bytes(1, 64, F16, F32) > 0
