"""The forms of the attention kernels that only larger calls reach, against the plain 64-bit implementation: prompts whose work
groups have eight waves, head sizes in between, and decode over rows so long that their page numbers are looked up in turns."""
import math

import pytest
import torch

import paper_2502_11880_amd as B
from tests import kv_model as M

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
WEIGHT = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -10}


def _announce(*what):
    print("case:", *what, flush=True)


def _check_prompts(b, H, new, io, seed, heads, window=0, sinks=0, rows=None):
    """Rows `rows` (positions from the end of each sequence's new tokens; None: all) of the given heads."""
    n, scale, D = sum(new), 1 / math.sqrt(b.dim), b.dim
    q = torch.randn(n, H * D, generator=torch.Generator().manual_seed(seed)).to(M.DTYPES[io])
    k, v, table, lens = b.on(DEV)
    start = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)
    out = torch.full((n, H * D), float("nan"), dtype=M.DTYPES[io], device=DEV)
    B.bitnet_attn_prefill(q.to(DEV), start.to(DEV), k, v, table, lens, out, scale, window, sinks)
    torch.cuda.synchronize()
    got, q, G = out.cpu().view(n, H, D), q.view(n, H, D), H // b.heads
    for s, m in enumerate(new):
        if m == 0:
            continue
        L, at = b.lens[s], int(start[s])
        i = torch.arange(m) if rows is None else torch.tensor(sorted({m - 1 - r for r in rows if r < m}))
        there = b.table[s].repeat_interleave(b.page)[:L]
        seen = M.visible(L - m + i, L, window, sinks) & ((there >= 0) & (there < b.pages))[None]
        for h in heads:
            want, tol = M.attention(q[at + i][:, h:h + 1], b.k[s][:, h // G:h // G + 1], b.v[s][:, h // G:h // G + 1], seen, scale,
                                    M.io_eps(io), WEIGHT[io])
            M.check(got[at + i][:, h:h + 1], want, tol, f"sequence {s}, head {h}")


# 32 kv heads and eight sequences and more: at least one work group of eight waves a CU, were all its columns used
@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 5), (33, 70)])
@pytest.mark.parametrize("dtype,io,H,D,page", [("f16", "f32", 32, 68, 16), ("f16", "f32", 32, 96, 64), ("f16", "f32", 64, 96, 16),
                                               ("f16", "f32", 32, 100, 32), ("f16", "f32", 32, 112, 128), ("f16", "f32", 32, 120, 16),
                                               ("f16", "f32", 96, 128, 256), ("bf16", "bf16", 32, 100, 16), ("f16", "f16", 32, 108, 64),
                                               ("bf16", "bf16", 64, 112, 32), ("f16", "f16", 32, 124, 16), ("bf16", "bf16", 32, 124, 64)])
def test_prompts_of_eight_waves(dtype, io, H, D, page, window, sinks):
    _announce("eight waves", dtype, io, H, D, page, window)
    new, past = [1, 300, 0, 64, 65, 7, 130, 257, 20], [0, 40, 9, 200, 0, 300, 77, 3, 500]
    b = M.Batch([n + p for n, p in zip(new, past)], 32, D, page, dtype, seed=D + page)
    b.table[7, 100 // page] = -1
    b.table[5, 0] = b.pages + 3
    _check_prompts(b, H, new, io, seed=51, heads=[0, H // 2 + 1, H - 1], window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,io,D,tokens,window", [("bf16", "bf16", 128, 2300, 0), ("f16", "f16", 128, 2300, 0), ("bf16", "bf16", 128, 3000, 2100),
                                                      ("f16", "f32", 128, 2300, 0), ("f16", "f32", 100, 2300, 700), ("bf16", "bf16", 100, 2300, 0),
                                                      ("f16", "f16", 96, 2300, 0), ("bf16", "f32", 128, 2300, 0)])
def test_long_prompts_of_many_heads(dtype, io, D, tokens, window):
    _announce("long prompt", dtype, io, D, tokens, window)
    b = M.Batch([tokens], 32, D, 64, dtype, seed=D + tokens)
    _check_prompts(b, 32, [tokens], io, seed=52, heads=[0, 17, 31], window=window, sinks=3 if window else 0,
                   rows=list(range(40)) + list(range(240, 275)) + [500, 701, 1023, 1024, 1500, 2040, 2200, 2298, 2299, 2999])


@pytest.mark.parametrize("dtype,io,D", [("f16", "f32", 96), ("f16", "f32", 100), ("bf16", "bf16", 104), ("f16", "f16", 124), ("f16", "f32", 128)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 4)])
def test_values_that_are_not_finite_in_eight_waves(dtype, io, D, window, sinks):
    _announce("eight waves, not finite", dtype, io, D, window)
    new = [290] + [40] * 8
    b = M.Batch(new, 32, D, 16, dtype, seed=D + 53)
    for head in (0, 20):
        b.v[0][100, head, 3] = float("nan")
        b.v[0][101, head, D - 4] = float("inf")
        b.v[0][150, head, D - 4] = float("-inf")
        b.v[0][0, head, 0] = float("inf")
        b.v[0][289, head, D - 1] = float("-inf")
        b.v[4][20, head, 60] = float("-inf")
    for s in (0, 4):
        b.write(s, 0, b.k[s], b.v[s])
    _check_prompts(b, 32, new, io, seed=53, heads=[0, 1, 20], window=window, sinks=sinks)


# head sizes between the sizes that the kernels are built for, four waves
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 4)])
@pytest.mark.parametrize("dtype,io,H,Hkv,D,page", [("bf16", "bf16", 4, 2, 72, 16), ("f16", "f16", 6, 2, 96, 64), ("bf16", "f32", 4, 1, 96, 32),
                                                   ("bf16", "bf16", 4, 4, 104, 128), ("f16", "f32", 4, 2, 112, 16), ("bf16", "f32", 3, 1, 108, 64),
                                                   ("bf16", "bf16", 8, 2, 124, 32), ("f16", "f16", 4, 1, 116, 256), ("bf16", "bf16", 5, 1, 144, 16),
                                                   ("f16", "f32", 2, 1, 192, 32), ("bf16", "f32", 2, 2, 200, 64), ("f16", "f16", 4, 1, 252, 16)])
def test_prompts_of_head_sizes_in_between(dtype, io, H, Hkv, D, page, window, sinks):
    _announce("head sizes", dtype, io, H, Hkv, D, page, window)
    new, past = [1, 150, 0, 64, 33], [0, 60, 4, 129, 700]
    b = M.Batch([n + p for n, p in zip(new, past)], Hkv, D, page, dtype, seed=D)
    b.table[4, 400 // page] = -1
    _check_prompts(b, H, new, io, seed=54, heads=list(range(H)), window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,io,H,D,page", [("bf16", "f32", 2, 64, 16), ("f16", "f16", 1, 64, 128), ("f16", "f32", 3, 40, 64), ("bf16", "bf16", 2, 128, 128)])
def test_decode_of_the_longest_rows(dtype, io, H, D, page):
    """One row of about 2^24 tokens that repeats the pages of 640: every work group's share is longer than the page numbers that it
    holds at a time.  The same output as over the 640 alone, since every one counts alike; some repetitions are missing."""
    _announce("decode 2^24", dtype, io, H, D, page)
    unique, most = 640, 1 << 24
    b = M.Batch([unique], 1, D, page, dtype, seed=D + page, spare=1)
    cycle = unique // page
    times = most // unique
    width = times * cycle
    table = b.table[:, :cycle].repeat(1, times)
    for gone in (0, 5, times // 2, times - 2):
        table[:, gone * cycle:(gone + 1) * cycle] = -1
    q = torch.randn(1, H * D, generator=torch.Generator().manual_seed(55)).to(M.DTYPES[io])
    k, v, _, _ = b.on(DEV)
    lens = torch.tensor([unique * times], dtype=torch.int32, device=DEV)
    need = B.bitnet_attn_decode_workspace_bytes(1, H, 1, D, page, width)
    out = torch.full((1, H * D), float("nan"), dtype=M.DTYPES[io], device=DEV)
    B.bitnet_attn_decode(q.to(DEV), k, v, table.contiguous().to(DEV), lens, out, 1 / math.sqrt(D), ws=torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    # sums run over a wave's quarter of a share (256 units of eight keys a lane), four waves, and a quarter of 512 parts: no more
    # additions in a row than the 640 keys that the tolerance counts
    want, tol = M.attention(q.view(1, H, D), b.k[0], b.v[0], torch.ones(1, unique, dtype=torch.bool), 1 / math.sqrt(D), M.io_eps(io),
                            2.0 ** -15 if io != "f32" else 0.0)
    M.check(out.view(1, H, D), want, tol)
