"""The paged key-value cache and the attention that reads it: what their speed is measured on.

A pass is one call (for the page operators: one short chain of calls) of the public entry points, or the same computation
as elementary torch operations in 32 bits (``own = False``).  Kinds of case:

* ``decode``  -- one new token per sequence over a paged cache (``bitnet_attn_decode``), with or without a sliding window
  and first tokens that stay visible;
* ``prefill`` -- the prompt tokens of a ragged batch, causal, behind whatever the cache already holds
  (``bitnet_attn_prefill``), with or without window and sinks;
* ``append``  -- the k and v products of new tokens written into their pages (``bitnet_kv_append``);
* ``fork``    -- a beam step: the old beams are freed, new ones forked from the survivors, each extended by one token
  (``bitnet_kv_free``, ``bitnet_kv_fork``, ``bitnet_kv_reserve``);
* ``compact`` -- a pool with holes moved to its lowest page numbers (``bitnet_kv_compact``).

Head counts and sizes are those of the 8B-class layer set (32 heads of 128 over 8 shared ones: the 4096 and 1024 rows of
its q and k/v) and of the 3B-class one (3200 rows: 32 heads of 100), and generic ones around them.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GOLDEN = 0.6180339887498949


def listed():
    return [
        # one user, a few words into a conversation: latency of a single call
        dict(name="decode-8b-b1-61", kind="decode", batch=1, length=61, ragged=False, heads=32, kv_heads=8, dim=128,
             cache="bf16", io="f32", page=16, window=0, sinks=0),
        # a serving batch of mixed lengths
        dict(name="decode-8b-b32-6000", kind="decode", batch=32, length=6000, ragged=True, heads=32, kv_heads=8, dim=128,
             cache="bf16", io="f32", page=32, window=0, sinks=0),
        # one user with a very long context: few rows, the length has to be split
        dict(name="decode-8b-b1-131071", kind="decode", batch=1, length=131071, ragged=False, heads=32, kv_heads=8,
             dim=128, cache="bf16", io="bf16", page=64, window=0, sinks=0),
        # long-running conversations with a sliding window and four first tokens; heads of 100
        dict(name="decode-3b-b24-window", kind="decode", batch=24, length=9000, ragged=True, heads=32, kv_heads=32,
             dim=100, cache="f16", io="f32", page=64, window=1024, sinks=4),
        # a one-sentence prompt
        dict(name="prefill-8b-37", kind="prefill", batch=1, tokens=37, past=0, ragged=False, heads=32, kv_heads=8, dim=128,
             cache="bf16", io="f32", page=16, window=0, sinks=0),
        # a long prompt
        dict(name="prefill-8b-4096", kind="prefill", batch=1, tokens=4096, past=0, ragged=False, heads=32, kv_heads=8,
             dim=128, cache="bf16", io="bf16", page=64, window=0, sinks=0),
        # chunks of several prompts behind what is already cached, window and sinks, heads of 100
        dict(name="prefill-3b-b6-window", kind="prefill", batch=6, tokens=1500, past=700, ragged=True, heads=32,
             kv_heads=32, dim=100, cache="f16", io="f32", page=32, window=512, sinks=4),
        # a document through a windowed layer
        dict(name="prefill-8b-8192-window", kind="prefill", batch=1, tokens=8192, past=0, ragged=False, heads=32,
             kv_heads=8, dim=128, cache="bf16", io="f32", page=128, window=1024, sinks=4),
        # one token of every sequence of a decode batch
        dict(name="append-8b-b64", kind="append", batch=64, tokens=1, past=500, ragged=True, heads=32, kv_heads=8, dim=128,
             cache="bf16", io="f32", page=32),
        # the k and v of several prompts
        dict(name="append-3b-b5-prompts", kind="append", batch=5, tokens=3000, past=100, ragged=True, heads=32,
             kv_heads=32, dim=100, cache="f16", io="f32", page=64),
        # a beam step of the 8B-class model: every layer's partial page copied
        dict(name="fork-8b-beams", kind="fork", layers=32, parents=8, fan=4, length=380, ragged=True, kv_heads=8, dim=128,
             cache="bf16", page=32),
        # a pool after many sequences came and went: half of its pages live
        dict(name="compact-8b", kind="compact", layers=32, pages=800, live=0.5, seqs=24, kv_heads=8, dim=128,
             cache="bf16", page=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges: one token to 131071, heads of 64 to 256 in steps of 4, one to 16 query heads for a
    shared one, every page size, both cache types, inputs in 32 bits or in the cache's type, windows and sinks."""
    kind = rng.choice(["decode"] * 4 + ["prefill"] * 3 + ["append"] * 2 + ["fork", "compact"])
    cache = rng.choice(["bf16", "f16"])
    page = rng.choice([16, 32, 64, 128, 256])
    case = dict(kind=kind, cache=cache, page=page, dim=rng.choice([64, 80, 96, 100, 112, 128, 128, 128, 192, 256]),
                kv_heads=rng.choice([1, 2, 4, 8, 8, 16, 32]))
    if kind in ("fork", "compact"):
        case["kv_heads"] = rng.choice([2, 4, 8])
        case["dim"] = rng.choice([64, 100, 128])
        case["layers"] = _log(rng, 1, 32)
        room = 32 * 32 * 8 * 128 // (case["layers"] * page * case["kv_heads"] * case["dim"])   # in pages of the listed cases
        if kind == "fork":
            case.update(parents=rng.randint(1, 8), fan=rng.randint(1, 4 if room >= 1 else 1), ragged=True)
            if case["parents"] * case["fan"] > 32 * max(room, 1):
                case["fan"] = 1
            case["length"] = _log(rng, 20, 380)
        else:
            case.update(pages=max(8, _log(rng, 64, max(64, min(4000, 790 * room)))), live=round(rng.uniform(0.2, 0.8), 2),
                        seqs=rng.randint(1, 32))
            while case["layers"] > 1 and case["pages"] * case["layers"] * page * case["kv_heads"] * case["dim"] > 790 * 32 * 32 * 1024:
                case["layers"] //= 2
        return case
    case["io"] = rng.choice(["f32", cache])
    group = rng.choice([1, 2, 3, 4, 4, 5, 8, 16])
    while group * case["kv_heads"] > 96:
        group = max(1, group // 2)
    case.update(heads=group * case["kv_heads"], ragged=rng.random() < 0.6)
    window = rng.random() < 0.4
    row = case["kv_heads"] * case["dim"]
    if kind == "decode":
        case.update(batch=_log(rng, 1, 64), length=_log(rng, 1, 131071))
        while case["batch"] * case["length"] * row > 100000 * 1024 or case["batch"] * case["length"] * case["heads"] > 1 << 22:
            if case["batch"] > 1 and rng.random() < 0.5:
                case["batch"] //= 2
            else:
                case["length"] = max(1, case["length"] // 2 + rng.randint(0, 7))
        case.update(window=_log(rng, 16, 4096) if window else 0, sinks=rng.randint(0, 70) if window else 0)
        return case
    if kind == "append":
        case.update(batch=_log(rng, 1, 128), tokens=1 if rng.random() < 0.5 else _log(rng, 2, 3000), past=_log(rng, 1, 500))
        while case["batch"] * (case["tokens"] + case["past"]) * row > 14000 * 3200:
            case["batch"], case["past"] = max(1, case["batch"] // 2), max(1, case["past"] // 2)
            case["tokens"] = max(1, case["tokens"] - case["tokens"] // 4)
        return case
    case.update(batch=_log(rng, 1, 12), tokens=_log(rng, 2, 4000), past=0 if rng.random() < 0.5 else _log(rng, 1, 4000))
    while case["batch"] * case["tokens"] * (case["tokens"] + case["past"]) * case["heads"] * case["dim"] > 0.45 * 4096 * 4096 * 4096:
        case["batch"] = max(1, case["batch"] // 2)
        case["tokens"], case["past"] = max(1, case["tokens"] * 3 // 4), case["past"] * 3 // 4
    case.update(window=_log(rng, 16, 2048) if window else 0, sinks=rng.randint(0, 70) if window else 0)
    return case


# ------------------------------------------------------------------------------------------------------------------
# Lengths of a case (by the case alone; the seed only orders the sequences)
# ------------------------------------------------------------------------------------------------------------------
def _spread(n, most, ragged):
    """n lengths from 1 to `most`: all `most`, or spread over the range with the first at its end."""
    if not ragged:
        return [most] * n
    return [1 + int((most - 1) * ((1 - b * GOLDEN) % 1 or 1.0)) for b in range(n)]


def _lengths(case):
    """(new tokens, cached tokens with the new ones) of every sequence."""
    if case["kind"] == "decode":
        return [1] * case["batch"], _spread(case["batch"], case["length"], case["ragged"])
    n = _spread(case["batch"], case["tokens"], case["ragged"])
    past = _spread(case["batch"], case["past"], case["ragged"])[::-1] if case["past"] else [0] * case["batch"]
    return n, [a + b for a, b in zip(n, past)]


def _visible(case, pos):
    """Keys that the query at position pos sees."""
    if not case["window"] or case["window"] > pos:
        return pos + 1
    return case["window"] + min(case["sinks"], pos + 1 - case["window"])


def _pairs(case):
    """(query, key) pairs in sight, and keys that some query sees, over the batch (one head)."""
    pairs = keys = 0
    for n, total in zip(*_lengths(case)):
        first = total - n
        if not case["window"]:
            pairs += n * first + n * (n + 1) // 2
            keys += total
        else:
            pairs += sum(_visible(case, p) for p in range(first, total))
            low = max(0, first + 1 - case["window"])
            keys += total - low + min(case["sinks"], low)
    return pairs, keys


def _chunks(dim):
    return -(-dim // 8)


def _page_bytes(case):
    """Bytes of one page's keys and of its values."""
    return case["kv_heads"] * case["page"] * _chunks(case["dim"]) * 16, case["kv_heads"] * case["page"] * case["dim"] * 2


def work(case):
    width = {"bf16": 2, "f16": 2, "f32": 4}
    kind = case["kind"]
    if kind in ("decode", "prefill"):
        pairs, keys = _pairs(case)
        n, total = _lengths(case)
        small = 8 * len(n) + 4 * sum(-(-t // case["page"]) for t in total)
        return {"bytes": keys * case["kv_heads"] * case["dim"] * 4 + 2 * sum(n) * case["heads"] * case["dim"] * width[case["io"]] + small,
                "flops": 4 * pairs * case["heads"] * case["dim"]}
    if kind == "append":
        n, _ = _lengths(case)
        return {"bytes": 2 * sum(n) * case["kv_heads"] * case["dim"] * (width[case["io"]] + 2), "flops": 0}
    k, v = _page_bytes(case)
    if kind == "fork":
        lens = _spread(case["parents"], case["length"], case["ragged"])
        moved = case["fan"] * sum(1 for t in lens if t % case["page"])
        entries = case["fan"] * sum(-(-t // case["page"]) for t in lens)
        return {"bytes": 2 * moved * case["layers"] * (k + v) + 16 * entries, "flops": 0}
    live = _live(case)
    # the pages that lie past the live count, of a live set spread evenly over the pool
    moved = live - round(live * live / case["pages"])
    return {"bytes": 2 * moved * case["layers"] * (k + v) + 8 * case["pages"], "flops": 0}


def _live(case):
    return min(case["pages"] - 1, max(1, int(case["pages"] * case["live"])))


# ------------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------------
def _pool(case, pages, gen, layers=None):
    """Keys [pages, Hkv, C, ps, 8] (zeros past dim) and values [pages, Hkv, ps / 8, dim, 8]: normal values, a few channels
    of the keys five times as large (with a leading dimension for the layers, if any)."""
    dt, h, d, ps, c = DTYPES[case["cache"]], case["kv_heads"], case["dim"], case["page"], _chunks(case["dim"])
    lead = (pages,) if layers is None else (layers, pages)
    k = torch.randn(*lead, h, c, ps, 8, dtype=dt, device=DEV, generator=gen)
    v = torch.randn(*lead, h, ps // 8, d, 8, dtype=dt, device=DEV, generator=gen)
    big = torch.rand(h, c, 1, 8, device=DEV, generator=gen) < 0.03
    gain = torch.where(big, 5.0, 1.0)
    gain.view(h, c, 8).masked_fill_((torch.arange(c * 8, device=DEV) >= d).view(1, c, 8), 0.0)
    return k.mul_(gain.to(dt)), v


def _sequences(case, gen):
    """Everything about the batch but its pages' contents: ordered lengths, the first token of each, the page table."""
    n, total = _lengths(case)
    order = torch.randperm(len(n), generator=gen, device=DEV)
    n = torch.tensor(n, dtype=torch.int32, device=DEV)[order]
    total_t = torch.tensor(total, dtype=torch.int32, device=DEV)[order]
    start = torch.zeros(len(total) + 1, dtype=torch.int32, device=DEV)
    start[1:] = torch.cumsum(n, 0)
    ps = case["page"]
    used = sum(-(-t // ps) for t in total)
    width = max(-(-t // ps) for t in total) + 1
    pages = used + 3
    ids = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    need = (total_t + ps - 1) // ps
    col = torch.arange(width, device=DEV)
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    table = torch.where(col < need[:, None], ids[at.clamp(max=pages - 1)], -1).to(torch.int32).contiguous()
    return start, total_t.contiguous(), table, pages


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "fork":
        return _prepare_fork(case, s, gen)
    if case["kind"] == "compact":
        return _prepare_compact(case, s, gen)
    start, total, table, pages = _sequences(case, gen)
    s.update(start=start, kv_len=total, table=table)
    s["k_cache"], s["v_cache"] = _pool(case, pages, gen)
    tokens = sum(_lengths(case)[0])
    io = DTYPES[case["io"]]
    if case["kind"] == "append":
        s["k"] = torch.randn(tokens, case["kv_heads"] * case["dim"], device=DEV, generator=gen).to(io)
        s["v"] = torch.randn(tokens, case["kv_heads"] * case["dim"], device=DEV, generator=gen).to(io)
        s["longest"] = max(_lengths(case)[0])
        return s
    s["q"] = torch.randn(tokens, case["heads"] * case["dim"], device=DEV, generator=gen).to(io)
    s["out"] = torch.empty_like(s["q"])
    s["scale"] = 1.0 / math.sqrt(case["dim"])
    s["longest"], s["past_most"] = max(_lengths(case)[0]), max(_lengths(case)[1])
    return s


def _prepare_fork(case, s, gen):
    lens = _spread(case["parents"], case["length"], case["ragged"])
    ps, nc = case["page"], case["parents"] * case["fan"]
    need = [-(-t // ps) for t in lens]
    width = max(need) + 2
    pages = sum(need) + 2 * nc + 5
    ids = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((case["parents"] + nc, width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, t in enumerate(need):
        table[i, :t] = ids[at:at + t]
        at += t
    kv_len = torch.zeros(case["parents"] + nc, dtype=torch.int32, device=DEV)
    kv_len[:case["parents"]] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[ids[:at].long()] = 1
    s["k_pool"], s["v_pool"] = _pool(case, pages, gen, case["layers"])
    child = torch.randperm(nc, generator=gen, device=DEV)
    s.update(table=table, kv_len=kv_len, refs=refs, children=(case["parents"] + child).to(torch.int32),
             parents=(torch.arange(nc, device=DEV) // case["fan"]).to(torch.int32),
             one=torch.ones(nc, dtype=torch.int32, device=DEV), short=torch.zeros(1, dtype=torch.int32, device=DEV))
    _plain_fork(s)                               # the beams of the step before
    return s


def _prepare_compact(case, s, gen):
    pages, live = case["pages"], _live(case)
    width = -(-live // case["seqs"])
    ids = torch.randperm(pages, generator=gen, device=DEV)[:live]
    table = torch.full((case["seqs"] * width,), -1, dtype=torch.int32, device=DEV)
    table[:live] = ids.to(torch.int32)
    refs = torch.zeros(pages, dtype=torch.int32, device=DEV)
    refs[ids] = 1
    s["k_pool"], s["v_pool"] = _pool(case, pages, gen, case["layers"])
    s.update(table0=table.view(case["seqs"], width), refs0=refs, n_live=torch.zeros(1, dtype=torch.int32, device=DEV))
    s["table"], s["refs"] = s["table0"].clone(), refs.clone()
    return s


# ------------------------------------------------------------------------------------------------------------------
# A pass
# ------------------------------------------------------------------------------------------------------------------
def run(state):
    s = state
    kind = s["kind"]
    if kind == "compact":                        # the holes of a pool in use
        s["table"].copy_(s["table0"])
        s["refs"].copy_(s["refs0"])
    (_own if own else _plain)[kind](s)
    if kind in ("decode", "prefill"):
        return s["out"] if own else s["plain"]
    if kind == "append":
        return [s["k_cache"], s["v_cache"]]
    if kind == "fork":
        return [s["k_pool"], s["v_pool"], s["table"], s["kv_len"], s["refs"], s["short"]]
    return [s["k_pool"], s["v_pool"], s["table"], s["refs"], s["n_live"]]


def _workspace(s, nbytes):
    """The workspace that a program keeps beside its cache."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes), dtype=torch.uint8, device=DEV)
    return s["ws"]


def _own_decode(s):
    import paper_2502_11880_amd as B
    ws = s["ws"] if "ws" in s else _workspace(s, B.bitnet_attn_decode_workspace_bytes(
        s["batch"], s["heads"], s["kv_heads"], s["dim"], s["page"], s["table"].shape[1], s["window"], s["sinks"]))
    B.bitnet_attn_decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["out"], s["scale"], s["window"],
                         s["sinks"], ws)


def _own_prefill(s):
    import paper_2502_11880_amd as B
    B.bitnet_attn_prefill(s["q"], s["start"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], s["out"], s["scale"],
                          s["window"], s["sinks"])


def _own_append(s):
    import paper_2502_11880_amd as B
    B.bitnet_kv_append(s["k"], s["v"], s["start"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"])


def _own_fork(s):
    import paper_2502_11880_amd as B
    ws = s["ws"] if "ws" in s else _workspace(s, B.bitnet_kv_workspace_bytes(s["refs"].shape[0], s["table"].shape[0]))
    B.bitnet_kv_free(s["table"], s["kv_len"], s["refs"], s["children"])
    B.bitnet_kv_fork(s["k_pool"], s["v_pool"], s["table"], s["kv_len"], s["refs"], s["parents"], s["children"], s["short"],
                     ws)
    B.bitnet_kv_reserve(s["table"], s["kv_len"], s["refs"], s["children"], s["one"], s["page"], s["short"], ws)


def _own_compact(s):
    import paper_2502_11880_amd as B
    ws = s["ws"] if "ws" in s else _workspace(s, B.bitnet_kv_workspace_bytes(s["refs"].shape[0], s["table"].shape[0]))
    B.bitnet_kv_compact(s["k_pool"], s["v_pool"], s["table"], s["refs"], s["n_live"], ws)


def _gather(s, longest):
    """Keys and values [B, Hkv, longest, dim] in 32 bits, read through the page table; zeros where the table has no page."""
    ps, h, d = s["page"], s["kv_heads"], s["dim"]
    cols = -(-longest // ps)
    table = s["table"][:, :cols]
    there = (table >= 0).repeat_interleave(ps, dim=1)[:, None, :longest, None]
    at = table.clamp(min=0).long()
    b = at.shape[0]
    k = s["k_cache"][at].permute(0, 2, 1, 4, 3, 5).reshape(b, h, cols * ps, -1)[:, :, :longest, :d].float()
    v = s["v_cache"][at].permute(0, 2, 1, 3, 5, 4).reshape(b, h, cols * ps, d)[:, :, :longest].float()
    return k * there, v * there


def _attend(q, k, v, seen, scale):
    """softmax(scale q k^T) v over the seen keys, zeros where none is: q [B, Hkv, rows, dim], seen [B, 1, rows, keys]."""
    b, h, r, d = q.shape
    x = torch.bmm(q.reshape(b * h, r, d), k.reshape(b * h, -1, d).transpose(1, 2).contiguous()).view(b, h, r, -1).mul_(scale)
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.bmm(x.view(b * h, r, -1), v.reshape(b * h, -1, d)).view(b, h, r, d)
    return torch.where(total > 0, y / total, 0.0)


def _seen(s, pos, keys):
    """Whether the query at position pos[...] sees each of the keys."""
    j = torch.arange(keys, device=DEV)
    p = pos[..., None]
    near = j <= p
    if not s["window"]:
        return near
    return near & ((j > p - s["window"]) | (j < s["sinks"]))


def _plain_decode(s):
    b, h, g, d = s["batch"], s["kv_heads"], s["heads"] // s["kv_heads"], s["dim"]
    longest = s["past_most"]
    k, v = _gather(s, longest)
    seen = _seen(s, s["kv_len"].long() - 1, longest)
    y = _attend(s["q"].float().view(b, h, g, d), k, v, seen[:, None, None, :].expand(b, 1, g, longest), s["scale"])
    s["plain"] = y.reshape(b, h * g * d).to(s["q"].dtype)


def _plain_prefill(s):
    b, h, g, d, n = s["batch"], s["kv_heads"], s["heads"] // s["kv_heads"], s["dim"], s["longest"]
    longest = s["past_most"]
    k, v = _gather(s, longest)
    start = s["start"].long()
    new = start[1:] - start[:-1]
    i = torch.arange(n, device=DEV)
    token = (start[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    pos = (s["kv_len"].long() - new)[:, None] + i
    seen = _seen(s, pos, longest) & (i < new[:, None])[..., None]
    q = s["q"][token].float().view(b, n, h, g, d).permute(0, 2, 1, 3, 4).reshape(b, h, n * g, d)
    rows = seen[:, None, :, None, :].expand(b, 1, n, g, longest).reshape(b, 1, n * g, longest)
    y = _attend(q, k, v, rows, s["scale"]).view(b, h, n, g, d).permute(0, 2, 1, 3, 4).reshape(b, n, h * g * d)
    at = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(start, at, right=True) - 1
    s["plain"] = y[seq, at - start[seq]].to(s["q"].dtype)


def _plain_append(s):
    h, d, ps = s["kv_heads"], s["dim"], s["page"]
    start = s["start"].long()
    at = torch.arange(s["k"].shape[0], device=DEV)
    seq = torch.searchsorted(start, at, right=True) - 1
    pos = s["kv_len"].long()[seq] - start[seq + 1] + at
    page, slot = s["table"][seq, pos // ps].long(), pos % ps
    k = s["k"].view(-1, h, d).to(s["k_cache"].dtype)
    k = torch.cat([k, k.new_zeros(k.shape[0], h, _chunks(d) * 8 - d)], 2) if d % 8 else k
    s["k_cache"][page, :, :, slot] = k.view(-1, h, _chunks(d), 8)
    s["v_cache"][page, :, slot // 8, :, slot % 8] = s["v"].view(-1, h, d).to(s["v_cache"].dtype)


def _count(refs, ids, by):
    """refs[id] += by for every id that is not -1."""
    more = torch.zeros(refs.shape[0] + 1, dtype=refs.dtype, device=refs.device)
    more.index_add_(0, torch.where(ids >= 0, ids, refs.shape[0]).reshape(-1).long(), torch.full((ids.numel(),), by, dtype=refs.dtype, device=refs.device))
    refs += more[:-1]


def _lowest_free(refs, count):
    """The `count` lowest free pages (the number of pages where there are none left)."""
    return torch.searchsorted(torch.cumsum(refs == 0, 0), torch.arange(1, count + 1, device=refs.device))


def _plain_fork(s):
    table, kv_len, refs, ps = s["table"], s["kv_len"], s["refs"], s["page"]
    kids, parents = s["children"].long(), s["parents"].long()
    n, width = kids.shape[0], table.shape[1]
    col = torch.arange(width, device=DEV)
    # free
    _count(refs, table[kids], -1)
    table[kids] = -1
    kv_len[kids] = 0
    # fork
    lens = kv_len[parents].long()
    full = lens // ps
    rows = torch.where(col < full[:, None], table[parents], -1)
    last = table[parents].gather(1, full.clamp(max=width - 1)[:, None])[:, 0]
    part = (lens % ps > 0) & (last >= 0)
    fresh = _lowest_free(refs, n)[(torch.cumsum(part, 0) - 1).clamp(min=0)].to(torch.int32)
    _count(refs, rows, 1)
    rows = torch.where((col == full[:, None]) & part[:, None], fresh[:, None], rows)
    table[kids] = rows
    kv_len[kids] = lens.to(torch.int32)
    _count(refs, torch.where(part, fresh, -1), 1)
    to, of = fresh[part].long(), last[part].long()
    s["k_pool"][:, to] = s["k_pool"][:, of]
    s["v_pool"][:, to] = s["v_pool"][:, of]
    # one token more for each
    lens = kv_len[kids].long() + s["one"]
    more = (lens + ps - 1) // ps > (lens - s["one"] + ps - 1) // ps
    fresh = _lowest_free(refs, n)[(torch.cumsum(more, 0) - 1).clamp(min=0)].to(torch.int32)
    at = (col == ((lens - 1) // ps)[:, None]) & more[:, None]
    table[kids] = torch.where(at, fresh[:, None], table[kids])
    kv_len[kids] = lens.to(torch.int32)
    _count(refs, torch.where(more, fresh, -1), 1)
    s["short"].zero_()                           # none went without a page


def _plain_compact(s):
    table, refs = s["table"], s["refs"]
    live = refs > 0
    count = live.sum()
    ids = torch.arange(refs.shape[0], device=DEV)
    to = (~live & (ids < count)).nonzero()[:, 0]
    of = (live & (ids >= count)).nonzero()[:, 0].flip(0)
    s["k_pool"][:, to] = s["k_pool"][:, of]
    s["v_pool"][:, to] = s["v_pool"][:, of]
    now = ids.to(torch.int32)
    now[of] = to.to(torch.int32)
    table.copy_(torch.where(table >= 0, now[table.clamp(min=0).long()], table))
    refs[to] = refs[of]
    refs[of] = 0
    s["n_live"].copy_(count)


_own = dict(decode=_own_decode, prefill=_own_prefill, append=_own_append, fork=_own_fork, compact=_own_compact)
_plain = dict(decode=_plain_decode, prefill=_plain_prefill, append=_plain_append, fork=_plain_fork, compact=_plain_compact)


# ------------------------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def _tokens_of(cache, row, count, value):
    """Tokens 0 .. count - 1 of one sequence, [count, Hkv, dim or the padded dim], in 64 bits, page by page."""
    ps = cache.shape[2] * 8 if value else cache.shape[3]
    got = []
    for page in row[:-(-count // ps)]:
        block = cache[page].double()             # keys [Hkv, C, ps, 8], values [Hkv, ps / 8, dim, 8]
        got.append(block.permute(1, 3, 0, 2).flatten(0, 1) if value else block.permute(2, 0, 1, 3).flatten(2))
    return torch.cat(got)[:count]


def exact(case, seed):
    if case["kind"] in ("fork", "compact"):
        return None                              # page numbers and copies
    s = prepare(case, seed)
    start, lens, table = s["start"].tolist(), s["kv_len"].tolist(), s["table"].tolist()
    h, d = case["kv_heads"], case["dim"]
    if case["kind"] == "append":
        keys, values = s["k_cache"].double(), s["v_cache"].double()
        k, v = s["k"].double().view(-1, h, d), s["v"].double().view(-1, h, d)
        for b, total in enumerate(lens):
            n, first = start[b + 1] - start[b], start[b]
            pos = torch.arange(total - n, total, device=DEV)
            page, slot = s["table"][b][pos // case["page"]].long(), pos % case["page"]
            for c in range(_chunks(d)):
                part = k[first:first + n, :, 8 * c:8 * c + 8]
                keys[page, :, c, slot, :part.shape[2]] = part
            values.transpose(3, 4)[page, :, slot // 8, slot % 8] = v[first:first + n]
        return [keys, values]
    g = case["heads"] // h
    out = torch.zeros(s["q"].shape[0], h, g, d, dtype=torch.float64, device=DEV)
    q = s["q"].double().view(-1, h, g, d)
    for b, total in enumerate(lens):
        first, n = (b, 1) if case["kind"] == "decode" else (start[b], start[b + 1] - start[b])
        pages = [p for p in table[b] if p >= 0]
        k, v = _tokens_of(s["k_cache"], pages, total, False), _tokens_of(s["v_cache"], pages, total, True)
        i = torch.arange(total - n, total, device=DEV)[:, None]
        j = torch.arange(total, device=DEV)[None, :]
        hidden = j > i
        if case["window"]:
            hidden |= (j <= i - case["window"]) & (j >= case["sinks"])
        for head in range(h):
            for r in range(g):
                x = q[first:first + n, head, r] @ k[:, head, :d].t() * s["scale"]
                p = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
                out[first:first + n, head, r] = p @ v[:, head]
    return out.view(s["q"].shape[0], -1)
