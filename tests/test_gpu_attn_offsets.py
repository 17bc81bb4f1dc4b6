"""Offsets of a ragged batch that do not start at 0, decrease, or lie outside the batch: rows that no sequence owns are left
alone, before the tensor, inside it and past it, and the sequences whose offsets hold get theirs."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _announce(*what):
    print("case:", *what, flush=True)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


# q_start, rows of the batch, cached tokens of each sequence, sequences whose rows have to be right
SPANS = [([64, 128], 128, [200], [0]), ([5, 5, 21, 40], 50, [9, 40, 19], [1, 2]), ([1000, 1010], 10, [30], []),
         ([0, 500, 20, 600], 600, [500, 40, 600], []), ([-2 ** 31, 5, 10], 10, [30, 30], [1]), ([300, 0, 100], 100, [300, 100], []),
         ([0, 2 ** 31 - 1, 7], 7, [9, 9], []), ([3, 9, 2 ** 31 - 1], 12, [6, 40], [0])]


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("start,rows,lens,right", SPANS)
def test_prefill_writes_only_rows_that_a_sequence_owns(start, rows, lens, right, split):
    _announce("prompt offsets", start, rows, split)
    H, Hkv, D, page, before = 32, 8, 64, 16, 1100
    b = M.Batch(lens, Hkv, D, page, "bf16", seed=rows, width=150)
    k, v, table, kv_len = b.on(DEV)
    q = torch.randn(rows, H * D, generator=torch.Generator().manual_seed(31))
    room = torch.full((before + rows + 300, H * D), 7.0, device=DEV)
    out = room[before:before + rows]
    need = B.bitnet_attn_prefill_workspace_bytes(1, 0, len(lens), rows, H, Hkv, D, page, table.shape[1])
    ws = torch.full((need + 16,), 0xFF, dtype=torch.uint8, device=DEV) if split else torch.empty(16, dtype=torch.uint8, device=DEV)
    B.bitnet_attn_prefill(q.to(DEV), _i32(start), k, v, table, kv_len, out, 1 / math.sqrt(D), ws=ws)
    torch.cuda.synchronize()
    owned = torch.zeros(rows, dtype=torch.bool)
    for s in range(len(lens)):
        if 0 <= start[s] <= start[s + 1] <= rows:
            owned[start[s]:start[s + 1]] = True
    assert bool((room[:before] == 7.0).all()), "rows before the tensor"
    assert bool((room[before + rows:] == 7.0).all()), "rows past the tensor"
    got = out.cpu()
    assert bool((got[~owned] == 7.0).all()), "rows that no sequence owns"
    for s in right:
        n, L = start[s + 1] - start[s], lens[s]
        want, tol = M.attention(q[start[s]:start[s + 1]].view(n, H, D), b.k[s], b.v[s], M.visible(torch.arange(L - n, L), L, 0, 0),
                                1 / math.sqrt(D), M.io_eps("f32"), 0.0)
        M.check(got[start[s]:start[s + 1]].view(n, H, D), want, tol, f"sequence {s}")


@pytest.mark.parametrize("start,rows,lens", [([64, 128], 128, [200]), ([512, 520], 600, [8]), ([9, 9, 30, 75], 80, [5, 33, 47]),
                                             ([600, 0, 90], 90, [20, 90]), ([-2 ** 31, 5, 10], 10, [30, 30]), ([0, 8, 16], 16, [2 ** 31 - 1, 20])])
def test_append_reads_only_its_sequences_rows_of_the_table(start, rows, lens):
    _announce("append offsets", start, rows, lens)
    H, D, page = 4, 64, 16
    held = [n if n < 10 ** 6 else 0 for n in lens]
    b = M.Batch(held, H, D, page, "f16", seed=rows, fill=0.5, width=20)
    kc, vc, table, _ = b.on(DEV)
    k, v = (torch.randn(rows, H, D, generator=torch.Generator().manual_seed(s)).to(b.dtype) for s in (32, 33))
    sure = []
    for s, n in enumerate(held):
        new = start[s + 1] - start[s]
        if start[s] >= 0 and 0 < new and start[s + 1] <= rows and n:
            sure.append(s)
            first = max(0, n - new)
            at = slice(start[s + 1] - (n - first), start[s + 1])
            b.write(s, first, k[at], v[at])
    B.bitnet_kv_append(k.to(DEV), v.to(DEV), _i32(start), kc, vc, table, _i32(lens))
    torch.cuda.synchronize()
    if start == sorted(start):               # offsets that decrease: what else is written is not said, only where
        assert torch.equal(kc.cpu(), b.k_cache) and torch.equal(vc.cpu(), b.v_cache)


@pytest.mark.parametrize("dtype,io,D", [("bf16", "bf16", 128), ("f16", "f32", 100), ("bf16", "f32", 64)])
@pytest.mark.parametrize("new,past", [([0] * 20 + [64] + [0] * 11, 1900), ([1] * 64, 1100), ([0, 3] * 40 + [90, 0, 0, 1], 700),
                                      ([0] * 700 + [70] + [0] * 200 + [2], 1500), ([0] * 1100 + [33], 1500)])
def test_prefill_of_tables_with_rows_that_have_no_tokens(new, past, dtype, io, D):
    """Split or not, however many rows of the table bring tokens: workspaces as the size query says, any contents."""
    _announce("sparse batch", len(new), sum(new), dtype, io, D)
    H, Hkv, page, n = 32, 8 if D == 128 else 32, 16, sum(new)
    b = M.Batch([c + past if c else (7 * i) % 40 for i, c in enumerate(new)], 1, D, page, dtype, seed=n + D, width=130)
    b.heads = Hkv                             # the same keys and values for every kv head
    k, v, table, kv_len = b.on(DEV)
    k, v = k.expand(-1, Hkv, -1, -1, -1).contiguous(), v.expand(-1, Hkv, -1, -1, -1).contiguous()
    start = torch.tensor([0] + new).cumsum(0).tolist()
    q = torch.randn(n, H * D, generator=torch.Generator().manual_seed(35)).to(M.DTYPES[io])
    kinds = {"f32": 0, "bf16": 1, "f16": 2}
    need = B.bitnet_attn_prefill_workspace_bytes(kinds[dtype], kinds[io], len(new), n, H, Hkv, D, page, 130)
    room = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device=DEV)
    out = torch.full((n, H * D), 7.0, dtype=M.DTYPES[io], device=DEV)
    B.bitnet_attn_prefill(q.to(DEV), _i32(start), k, v, table, kv_len, out, 0.1, ws=room[:need] if need else room[:16])
    torch.cuda.synchronize()
    assert bool((room[need:] == 0xFF).all()), "bytes past the workspace"
    got = out.cpu().view(n, H, D)
    weight = 0.0 if io == "f32" else {"bf16": 2.0 ** -8, "f16": 2.0 ** -10}[io]
    for s in [i for i, c in enumerate(new) if c][:6] + [i for i, c in enumerate(new) if c][-3:]:
        L, rows = b.lens[s], slice(start[s], start[s + 1])
        for heads in (slice(0, 2), slice(H - 2, H)):
            want, tol = M.attention(q[rows].view(-1, H, D)[:, heads], b.k[s], b.v[s], M.visible(torch.arange(L - new[s], L), L, 0, 0),
                                    0.1, M.io_eps(io), weight)
            M.check(got[rows, heads], want, tol, f"sequence {s}")
