"""What stands between the products of a served layer: what its speed is measured on.

A pass is one call of the public entry points, or the same computation as elementary torch operations (``own = False``).
Kinds of case:

* ``norm``   -- the residual's addition, the root-mean-square norm and the int8 codes that the next product reads
  (``bitnet_norm_quantize``);
* ``rope``   -- the position rotation of query heads (``bitnet_rope``);
* ``append`` -- keys rotated by their positions and written with the values into their pages, the query heads rotated on the
  way (``bitnet_kv_append_rope``);
* ``shared`` -- one new token per sequence over a paged cache in which groups of sequences share a long prefix
  (``bitnet_attn_decode_shared``), with or without a sliding window and first tokens that stay visible.

Head counts and sizes are those of the 8B-class layer set (32 heads of 128 over 8 shared ones, rows of 4096) and of the
3B-class one (32 heads of 100, rows of 3200 and 8640), and generic ones around them.

The codes of ``norm`` are the integers that the next product multiplies; its definition rounds to 32 bits at stated places
only, so codes, scales and sums have one right value each.
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
GOLDEN = 0.6180339887498949
EPS = 1e-5


def listed():
    return [
        # one token's hidden state before q/k/v: latency of a single call
        dict(name="norm-8b-1", kind="norm", rows=1, width=4096, x="f32", residual="f32"),
        # a chunk of prompts before the down product, the stream in 16 bits; rows of no power of two
        dict(name="norm-3b-333", kind="norm", rows=333, width=8640, x="f32", residual="bf16"),
        # a large prefill
        dict(name="norm-8b-8192", kind="norm", rows=8192, width=4096, x="f32", residual="f32"),
        # the query heads of a few sequences at far positions
        dict(name="rope-8b-7", kind="rope", tokens=7, heads=32, dim=128, rot=128, io="f32", interleaved=False, far=1 << 20,
             scaling="none"),
        # a batch of prompts, less than half of the head rotated in pairs of neighbours
        dict(name="rope-3b-6001", kind="rope", tokens=6001, heads=32, dim=100, rot=48, io="f16", interleaved=True, far=8192,
             scaling="linear"),
        # one token of every sequence of a decode batch
        dict(name="append-8b-b64", kind="append", batch=64, tokens=1, past=8000, ragged=True, heads=32, kv_heads=8, dim=128,
             rot=128, cache="bf16", io="f32", page=32, interleaved=False, scaling="turns"),
        # several prompts of mixed lengths, frequencies stretched for a long context
        dict(name="append-8b-b5-prompts", kind="append", batch=5, tokens=3001, past=100, ragged=True, heads=32, kv_heads=8,
             dim=128, rot=128, cache="bf16", io="f32", page=64, interleaved=False, scaling="index"),
        # chunks behind what is cached, heads of 100 of which 64 channels turn
        dict(name="append-3b-b9-chunks", kind="append", batch=9, tokens=509, past=2000, ragged=True, heads=32, kv_heads=32,
             dim=100, rot=64, cache="f16", io="f16", page=16, interleaved=True, scaling="none"),
        # four beams a few hundred tokens into an answer
        dict(name="shared-8b-beams4", kind="shared", groups=1, members=4, prefix=352, tail=40, ragged=True, heads=32, kv_heads=8,
             dim=128, cache="bf16", io="f32", page=32, window=0, sinks=0),
        # a serving batch behind one system prompt, each with a conversation of its own
        dict(name="shared-8b-b32-6016", kind="shared", groups=1, members=32, prefix=6016, tail=1500, ragged=True, heads=32,
             kv_heads=8, dim=128, cache="bf16", io="f32", page=32, window=0, sinks=0),
        # several groups of different sizes, heads of 100 with keys of their own
        dict(name="shared-3b-g5", kind="shared", groups=5, members=12, prefix=5003, tail=600, ragged=True, heads=32, kv_heads=32,
             dim=100, cache="f16", io="f32", page=64, window=0, sinks=0),
        # many questions about one long document
        dict(name="shared-8b-b64-65536", kind="shared", groups=1, members=64, prefix=65536, tail=257, ragged=True, heads=32,
             kv_heads=8, dim=128, cache="bf16", io="bf16", page=64, window=0, sinks=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges: one row to 8192 of 64 to 16384 values; one token to 6001; heads of 64 to 256 in steps of 4,
    all or part of them rotated, both layouts of pairs and every scaling; one to eight groups of one to 64 sequences with
    prefixes of up to 65536 tokens; every page size, both cache types, inputs in 32 bits or in 16, windows and sinks."""
    kind = rng.choice(["norm"] * 3 + ["rope"] * 2 + ["append"] * 3 + ["shared"] * 4)
    if kind == "norm":
        wide = rng.choice(["f32", "bf16", "f16"])
        case = dict(kind=kind, rows=_log(rng, 1, 8192), width=_log(rng, 64, 16384), residual=rng.choice([wide, wide, ""]),
                    x=rng.choice(["f32", wide]))
        if rng.random() < 0.6:
            case["width"] = max(64, case["width"] // 64 * 64)
        while case["rows"] * case["width"] > 8192 * 4096:
            case["rows"] = max(1, case["rows"] * 3 // 4)
        return case
    dim = rng.choice([64, 80, 96, 100, 112, 128, 128, 128, 192, 256])
    if kind != "shared":
        turn = dict(rot=rng.choice([dim, dim, dim // 2 // 2 * 2, dim * 3 // 4 // 2 * 2]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "base", "turns", "index"]))
    if kind == "rope":
        case = dict(kind=kind, tokens=_log(rng, 1, 6001), heads=rng.choice([1, 2, 5, 8, 16, 32, 64]), dim=dim,
                    io=rng.choice(["f32", "bf16", "f16"]), far=_log(rng, 64, 1 << 23), **turn)
        while case["tokens"] * case["heads"] * dim > 6001 * 3200:
            case["tokens"] = max(1, case["tokens"] // 2)
        return case
    cache = rng.choice(["bf16", "f16"])
    case = dict(kind=kind, cache=cache, page=rng.choice([16, 32, 64, 128, 256]), dim=dim, kv_heads=rng.choice([1, 2, 4, 8, 8, 16, 32]),
                io=rng.choice(["f32", cache]), ragged=rng.random() < 0.6)
    per = rng.choice([1, 2, 3, 4, 4, 5, 8, 16])
    while per * case["kv_heads"] > 64:
        per = max(1, per // 2)
    case["heads"] = per * case["kv_heads"]
    if kind == "append":
        case.update(batch=_log(rng, 1, 128), tokens=1 if rng.random() < 0.5 else _log(rng, 2, 3001), past=_log(rng, 1, 8000), **turn)
        while case["batch"] * case["tokens"] * (case["heads"] + 2 * case["kv_heads"]) * dim > 5 * 1500 * 48 * 128 or \
                case["batch"] * (case["past"] + case["tokens"]) * case["kv_heads"] * dim > 64 * 4000 * 8 * 128:
            case["batch"], case["past"] = max(1, case["batch"] // 2), max(1, case["past"] // 2)
            case["tokens"] = max(1, case["tokens"] - case["tokens"] // 4)
        return case
    case.update(groups=_log(rng, 1, 8), members=_log(rng, 1, 64), prefix=_log(rng, 1, 65536), tail=_log(rng, 1, 1500))
    while case["groups"] * case["members"] > 64:
        case["groups"], case["members"] = max(1, case["groups"] // 2), max(1, case["members"] * 3 // 4)
    while case["groups"] * case["members"] * (case["prefix"] + case["tail"]) * case["heads"] * dim > 64 * 65536 * 32 * 128 // 4 or \
            case["groups"] * (case["prefix"] + case["members"] * case["tail"]) * case["kv_heads"] * dim > 65536 * 8 * 128:
        case["prefix"] = max(1, case["prefix"] * 3 // 4)
        case["tail"] = max(1, case["tail"] * 7 // 8)
    if rng.random() < 0.5:
        case["prefix"] = -(-case["prefix"] // case["page"]) * case["page"]
    window = rng.random() < 0.25
    case.update(window=_log(rng, 16, 4096) if window else 0, sinks=rng.randint(0, 70) if window else 0)
    return case


# ------------------------------------------------------------------------------------------------------------------
# Lengths of a case (by the case alone; the seed only orders the sequences)
# ------------------------------------------------------------------------------------------------------------------
def _spread(n, most, ragged):
    """n lengths from 1 to `most`: all `most`, or spread over the range with the first at its end."""
    if not ragged:
        return [most] * n
    return [1 + int((most - 1) * ((1 - b * GOLDEN) % 1 or 1.0)) for b in range(n)]


def _append_lengths(case):
    """(new tokens, cached tokens with the new ones) of every sequence."""
    n = _spread(case["batch"], case["tokens"], case["ragged"])
    past = _spread(case["batch"], case["past"], case["ragged"])[::-1]
    return n, [a + b for a, b in zip(n, past)]


def _groups(case):
    """(members, prefix) of every group, and the tokens behind the prefix of every sequence in the order of the groups."""
    members = _spread(case["groups"], case["members"], case["ragged"])
    prefix = _spread(case["groups"], case["prefix"], case["ragged"])
    return list(zip(members, prefix)), _spread(sum(members), case["tail"], case["ragged"])


def _behind(case, length):
    """First key of the window of the last of `length` tokens."""
    return max(0, length - case["window"]) if case["window"] else 0


def _shared_pairs(case):
    """(query, key) pairs in sight and keys that some query sees, of one head."""
    groups, tails = _groups(case)
    pairs = keys = at = 0
    for members, prefix in groups:
        lows = []
        for tail in tails[at:at + members]:
            low = _behind(case, prefix + tail)
            lows.append(low)
            pairs += prefix + tail - low + min(case["sinks"], low)
            keys += prefix + tail - max(low, prefix) + max(0, min(case["sinks"], low) - prefix)
        at += members
        low = min(min(lows), prefix)
        keys += prefix - low + min(case["sinks"], low)
    return pairs, keys


def _chunks(dim):
    return -(-dim // 8)


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4, "": 0}
    if case["kind"] == "norm":
        values = case["rows"] * case["width"]
        return {"bytes": values * (size[case["x"]] + 2 * size[case["residual"]] + 1) + 4 * case["width"] + 8 * case["rows"],
                "flops": 8 * values}
    if case["kind"] == "rope":
        rows = case["tokens"] * case["heads"]
        return {"bytes": 2 * rows * case["dim"] * size[case["io"]] + 4 * case["tokens"] + 4 * case["rot"], "flops": 3 * rows * case["rot"]}
    if case["kind"] == "append":
        n, total = _append_lengths(case)
        pages = sum(-(-t // case["page"]) - (t - a) // case["page"] for a, t in zip(n, total))
        return {"bytes": sum(n) * case["dim"] * (2 * case["heads"] * size[case["io"]] + 2 * case["kv_heads"] * (size[case["io"]] + 2)) + 8 * len(n) + 4 * pages,
                "flops": 3 * sum(n) * (case["heads"] + case["kv_heads"]) * case["rot"]}
    pairs, keys = _shared_pairs(case)
    groups, tails = _groups(case)
    small = 4 * len(tails) + 8 * len(groups) + 4 * (keys // case["page"])
    return {"bytes": keys * case["kv_heads"] * case["dim"] * 4 + 2 * len(tails) * case["heads"] * case["dim"] * size[case["io"]] + small,
            "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------------
THETA, FACTOR, ORIGINAL = 10000.0, 8.0, 4096


def _frequencies(case):
    """Turns a position of each pair, in 64 bits on the host: theta^(-2i / rot) / 2 pi, stretched by a factor: everywhere
    (linear), by a larger theta (base), or where a pair makes few turns over the original context: below 1 fully, above 4 (turns)
    or 32 (index: the border in the pairs' index) not at all."""
    r, kind = case["rot"], case["scaling"]
    theta = THETA * (FACTOR ** (r / (r - 2)) if kind == "base" else 1.0)
    f = [theta ** (-2.0 * i / r) / (2 * math.pi) for i in range(r // 2)]
    if kind == "linear":
        return [x / FACTOR for x in f]
    if kind == "turns":
        keep = [min(1.0, max(0.0, (ORIGINAL * x - 1.0) / (4.0 - 1.0))) for x in f]
    elif kind == "index":
        border = [r * math.log(ORIGINAL / (t * 2 * math.pi)) / (2 * math.log(THETA)) for t in (32.0, 1.0)]
        lo, hi = max(0, math.floor(border[0])), min(r - 1, math.ceil(border[1]))
        keep = [1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001))) for i in range(r // 2)]
    else:
        return f
    return [x * w + x / FACTOR * (1.0 - w) for x, w in zip(f, keep)]


def _gain(case):
    return 1.0 + 0.1 * math.log(FACTOR) if case["scaling"] == "index" else 1.0


def _pool(case, pages, gen):
    """Keys [pages, Hkv, C, ps, 8] (zeros past dim) and values [pages, Hkv, ps / 8, dim, 8]: normal values, a few channels
    of the keys five times as large."""
    dt, h, d, ps, c = DTYPES[case["cache"]], case["kv_heads"], case["dim"], case["page"], _chunks(case["dim"])
    k = torch.randn(pages, h, c, ps, 8, dtype=dt, device=DEV, generator=gen)
    v = torch.randn(pages, h, ps // 8, d, 8, dtype=dt, device=DEV, generator=gen)
    big = torch.rand(h, c, 1, 8, device=DEV, generator=gen) < 0.03
    gain = torch.where(big, 5.0, 1.0)
    gain.view(h, c, 8).masked_fill_((torch.arange(c * 8, device=DEV) >= d).view(1, c, 8), 0.0)
    return k.mul_(gain.to(dt)), v


def _rows(shape, io, gen):
    """Rows as products leave them: normal values, some channels several times as large as others."""
    x = torch.randn(*shape, device=DEV, generator=gen)
    return x.mul_(torch.exp(0.7 * torch.randn(shape[-1], device=DEV, generator=gen))).to(DTYPES[io])


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "norm":
        m, k = case["rows"], case["width"]
        s["in"] = _rows((m, k), case["x"], gen)
        s["gamma"] = 1.0 + 0.2 * torch.randn(k, device=DEV, generator=gen)
        if case["residual"]:
            s["res"] = _rows((m, k), case["residual"], gen).mul_(3.0)
            s["res_out"] = torch.empty_like(s["res"])
        s["xq"] = torch.empty(m, k, dtype=torch.int8, device=DEV)
        s["x_scale"] = torch.empty(m, device=DEV)
        s["x_rowsum"] = torch.empty(m, dtype=torch.int32, device=DEV)
        return s
    if case["kind"] == "rope":
        s["in"] = _rows((case["tokens"], case["heads"] * case["dim"]), case["io"], gen)
        s["pos"] = torch.randint(0, case["far"], (case["tokens"],), dtype=torch.int32, device=DEV, generator=gen)
        s["turns"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
        s["out"] = torch.empty_like(s["in"])
        return s
    if case["kind"] == "append":
        return _prepare_append(case, s, gen)
    return _prepare_shared(case, s, gen)


def _prepare_append(case, s, gen):
    n, total = _append_lengths(case)
    order = torch.randperm(len(n), generator=gen, device=DEV).tolist()
    n, total = [n[i] for i in order], [total[i] for i in order]
    ps = case["page"]
    need = [-(-t // ps) for t in total]
    pages = sum(need) + 3
    ids = torch.randperm(pages, generator=gen, device=DEV).tolist()
    rows, at, start = [], 0, [0]
    for b, t in enumerate(need):
        rows.append(ids[at:at + t] + [-1] * (max(need) + 1 - t))
        at += t
        start.append(start[-1] + n[b])
    s.update(table=_ints(rows), kv_len=_ints(total), start=_ints(start))
    s["k_cache"], s["v_cache"] = _pool(case, pages, gen)
    io, d = case["io"], case["dim"]
    s["q"] = _rows((start[-1], case["heads"] * d), io, gen)
    s["k"] = _rows((start[-1], case["kv_heads"] * d), io, gen)
    s["v"] = torch.randn(start[-1], case["kv_heads"] * d, device=DEV, generator=gen).to(DTYPES[io])
    s["q_out"] = torch.empty_like(s["q"])
    s["turns"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
    return s


def _prepare_shared(case, s, gen):
    groups, tails = _groups(case)
    ps = case["page"]
    order = torch.randperm(len(tails), generator=gen, device=DEV).tolist()
    tails = [tails[i] for i in order]
    width = max(-(-(p + case["tail"]) // ps) for _, p in groups) + 1
    need = sum(-(-p // ps) for _, p in groups) + sum(-(-t // ps) + 1 for t in tails)
    ids = torch.randperm(need + 3, generator=gen, device=DEV).tolist()
    rows, lens, start, at, b = [], [], [0], 0, 0
    for members, prefix in groups:                # whole pages of the prefix in every member's row, the rest of its own
        full = prefix // ps
        common = ids[at:at + full]
        first = ids[at + full:at + full + 1] if prefix % ps else []
        at += full + len(first)
        for i in range(members):
            total = prefix + tails[b]
            mine = -(-total // ps) - full
            if i == 0 and first:
                row = common + first + ids[at:at + mine - 1]
                at += mine - 1
            else:
                row = common + ids[at:at + mine]
                at += mine
            rows.append(row + [-1] * (width - len(row)))
            lens.append(total)
            b += 1
        start.append(b)
    s.update(table=_ints(rows), kv_len=_ints(lens), group_start=_ints(start), prefix_len=_ints([p for _, p in groups]))
    s["k_cache"], s["v_cache"] = _pool(case, need + 3, gen)
    for g, (members, prefix) in enumerate(groups):   # a last page of the prefix that is not full: every member's own copy
        if prefix % ps == 0:
            continue
        src = rows[start[g]][prefix // ps]
        for b in range(start[g] + 1, start[g + 1]):
            dst, part = rows[b][prefix // ps], prefix % ps
            s["k_cache"][dst, :, :, :part] = s["k_cache"][src, :, :, :part]
            v = s["v_cache"].transpose(3, 4)
            full, rest = part // 8, part % 8
            v[dst, :, :full] = v[src, :, :full]
            if rest:
                v[dst, :, full, :rest] = v[src, :, full, :rest]
    s["lens"], s["starts"], s["prefixes"] = lens, start, [p for _, p in groups]
    s["q"] = torch.randn(len(lens), case["heads"] * case["dim"], device=DEV, generator=gen).to(DTYPES[case["io"]])
    s["out"] = torch.empty_like(s["q"])
    s["scale"] = 1.0 / math.sqrt(case["dim"])
    return s


# ------------------------------------------------------------------------------------------------------------------
# A pass
# ------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_own if own else _plain)[state["kind"]](state)


def _own_norm(s):
    import paper_2502_11880_amd as B
    B.bitnet_norm_quantize(s["in"], s["gamma"], EPS, s["xq"], s["x_scale"], s["x_rowsum"], s.get("res"), s.get("res_out"))
    return [s["xq"], s["x_scale"], s["x_rowsum"]] + ([s["res_out"]] if s["residual"] else [])


def _own_turns(s):
    """The frequencies that a program keeps beside its model."""
    if "freqs" not in s:
        import paper_2502_11880_amd as B
        s["freqs"] = torch.empty(s["rot"] // 2, dtype=torch.float64, device=DEV)
        low, high = (1.0, 4.0) if s["scaling"] == "turns" else (1.0, 32.0)
        B.bitnet_rope_freqs(s["freqs"], THETA, s["scaling"], FACTOR, ORIGINAL, low, high)
    return s["freqs"]


def _own_rope(s):
    import paper_2502_11880_amd as B
    B.bitnet_rope(s["in"], s["pos"], _own_turns(s), s["out"], s["dim"], s["interleaved"], _gain(s))
    return s["out"]


def _own_append(s):
    import paper_2502_11880_amd as B
    B.bitnet_kv_append_rope(s["k"], s["v"], s["start"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"], _own_turns(s),
                            s["interleaved"], _gain(s), s["q"], s["q_out"])
    return [s["q_out"], s["k_cache"], s["v_cache"]]


def _own_shared(s):
    import paper_2502_11880_amd as B
    if "ws" not in s:                            # the workspace that a program keeps beside its cache
        need = B.bitnet_attn_decode_shared_workspace_bytes(len(s["lens"]), s["heads"], s["kv_heads"], s["dim"], s["page"],
                                                           s["table"].shape[1], s["window"], s["sinks"])
        s["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device=DEV)
    B.bitnet_attn_decode_shared(s["q"], s["group_start"], s["prefix_len"], s["k_cache"], s["v_cache"], s["table"], s["kv_len"],
                                s["out"], s["scale"], s["window"], s["sinks"], s["ws"])
    return s["out"]


def _plain_norm(s):
    r = s["in"].float()
    if s["residual"]:
        s["res_out"] = (r + s["res"].float()).to(s["res"].dtype)
        r = s["res_out"].float()
    inv = (1.0 / torch.sqrt((r.double() * r.double()).sum(1, keepdim=True) / s["width"] + EPS)).float()
    n = r * inv * s["gamma"]
    scale = (127.0 / n.abs().amax(1).clamp(min=1e-5).double()).float()
    codes = torch.round(n * scale[:, None]).clamp(-128, 127).to(torch.int8)
    return [codes, scale, codes.sum(1, dtype=torch.int32)] + ([s["res_out"]] if s["residual"] else [])


def _turn(s, x, pos):
    """x [tokens, heads, dim] in 32 bits with its first channels rotated by the angles of pos (in 64 bits)."""
    r = s["rot"]
    angle = pos.double()[:, None] * s["turns"]
    angle = (angle - torch.round(angle)) * (2 * math.pi)
    c, z = (torch.cos(angle) * _gain(s)).float()[:, None], (torch.sin(angle) * _gain(s)).float()[:, None]
    out = x.clone()
    a, b = (slice(0, r, 2), slice(1, r, 2)) if s["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    out[..., a] = x[..., a] * c - x[..., b] * z
    out[..., b] = x[..., b] * c + x[..., a] * z
    return out


def _plain_rope(s):
    x = s["in"].float().view(s["tokens"], s["heads"], s["dim"])
    return _turn(s, x, s["pos"]).reshape(s["in"].shape).to(s["in"].dtype)


def _plain_append(s):
    h, d, ps = s["kv_heads"], s["dim"], s["page"]
    start = s["start"].long()
    at = torch.arange(s["k"].shape[0], device=DEV)
    seq = torch.searchsorted(start, at, right=True) - 1
    pos = s["kv_len"].long()[seq] - start[seq + 1] + at
    page, slot = s["table"][seq, pos // ps].long(), pos % ps
    q = _turn(s, s["q"].float().view(-1, s["heads"], d), pos).reshape(s["q"].shape).to(s["q"].dtype)
    k = _turn(s, s["k"].float().view(-1, h, d), pos).to(s["k_cache"].dtype)
    k = torch.cat([k, k.new_zeros(k.shape[0], h, _chunks(d) * 8 - d)], 2) if d % 8 else k
    s["k_cache"][page, :, :, slot] = k.view(-1, h, _chunks(d), 8)
    s["v_cache"][page, :, slot // 8, :, slot % 8] = s["v"].view(-1, h, d).to(s["v_cache"].dtype)
    return [q, s["k_cache"], s["v_cache"]]


def _gather(s, rows, first, last):
    """Keys and values [rows, Hkv, last - first, dim] of positions first .. last - 1 in 32 bits, read through table rows."""
    h, d = s["kv_heads"], s["dim"]
    pos = torch.arange(first, last, device=DEV)
    page, slot = rows[:, pos // s["page"]].long().clamp(min=0), (pos % s["page"]).expand(rows.shape[0], -1)
    k = s["k_cache"].permute(0, 3, 1, 2, 4)[page, slot].reshape(*page.shape, h, -1)[..., :d]
    v = s["v_cache"].permute(0, 2, 4, 1, 3)[page, slot // 8, slot % 8]
    return k.float().transpose(1, 2).contiguous(), v.float().transpose(1, 2).contiguous()


def _scores(s, q, k, seen):
    """scale q k^T over the seen keys, -inf elsewhere: q [n, Hkv, rows, dim], k [n, Hkv, keys, dim], seen [n, 1, rows, keys]."""
    n, h, r, d = q.shape
    x = torch.bmm(q.reshape(n * h, r, d), k.reshape(n * h, -1, d).transpose(1, 2).contiguous()).view(n, h, r, -1)
    return x.mul_(s["scale"]).masked_fill_(~seen, -math.inf)


def _weighted(p, v):
    n, h, r, keys = p.shape
    return torch.bmm(p.reshape(n * h, r, keys), v.reshape(n * h, keys, -1)).view(n, h, r, -1)


def _plain_shared(s):
    h, g, d = s["kv_heads"], s["heads"] // s["kv_heads"], s["dim"]
    out = torch.empty_like(s["q"])
    for i, prefix in enumerate(s["prefixes"]):
        b0, b1 = s["starts"][i], s["starts"][i + 1]
        m, longest = b1 - b0, max(s["lens"][b0:b1])
        q = s["q"][b0:b1].float().view(m, h, g, d)
        lens = s["kv_len"][b0:b1].long()[:, None]
        j = torch.arange(longest, device=DEV)[None]
        seen = j < lens
        if s["window"]:
            seen = seen & ((j >= lens - s["window"]) | (j < s["sinks"]))
        k0, v0 = _gather(s, s["table"][b0:b0 + 1], 0, prefix)
        k1, v1 = _gather(s, s["table"][b0:b1], prefix, longest)
        q0 = q.permute(1, 0, 2, 3).reshape(1, h, m * g, d)
        seen0 = seen[:, None, :prefix].expand(m, g, prefix).reshape(1, 1, m * g, prefix)
        x0 = _scores(s, q0, k0, seen0)
        x1 = _scores(s, q, k1, seen[:, None, None, prefix:].expand(m, 1, g, longest - prefix))
        top0 = x0.amax(-1).view(h, m, g).permute(1, 0, 2)
        top = torch.maximum(top0, x1.amax(-1))
        top = torch.where(top == -math.inf, 0.0, top)
        x0 = x0.sub_(top.permute(1, 0, 2).reshape(1, h, m * g, 1)).exp_()
        x1 = x1.sub_(top[..., None]).exp_()
        total = x0.sum(-1).view(h, m, g).permute(1, 0, 2) + x1.sum(-1)
        y = _weighted(x0, v0).view(h, m, g, d).permute(1, 0, 2, 3) + _weighted(x1, v1)
        out[b0:b1] = torch.where(total[..., None] > 0, y / total[..., None], 0.0).reshape(m, h * g * d).to(out.dtype)
    return out


_own = dict(norm=_own_norm, rope=_own_rope, append=_own_append, shared=_own_shared)
_plain = dict(norm=_plain_norm, rope=_plain_rope, append=_plain_append, shared=_plain_shared)


# ------------------------------------------------------------------------------------------------------------------
# The definition in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def _exact_norm(s):
    """Row by row from the formulas, rounded to 32 bits where the definition says so (and to the residual's type)."""
    r = s["in"].double()
    outs = []
    if s["residual"]:
        outs = [(r + s["res"].double()).float().to(s["res"].dtype)]
        r = outs[0].double()
    inv = ((r.pow(2).mean(1) + EPS) ** -0.5).float().double()
    n = ((r * inv[:, None]).float().double() * s["gamma"].double()).float().double()
    top = n.abs().max(1).values
    scale = (127.0 / torch.maximum(top, torch.full_like(top, 1e-5).float().double())).float()
    codes = torch.round((n * scale.double()[:, None]).float()).clamp(-128.0, 127.0)
    return [codes.to(torch.int8), scale, codes.double().sum(1).to(torch.int32)] + outs


def _exact_turn(s, x, pos):
    """The rotation as a product of complex numbers."""
    r = s["rot"]
    turns = torch.tensor(_frequencies(s), dtype=torch.float64, device=DEV)
    f = torch.polar(torch.full((pos.shape[0], r // 2), _gain(s), dtype=torch.float64, device=DEV),
                    torch.remainder(pos.double()[:, None] * turns, 1.0) * (2 * math.pi))[:, None, :]
    head = x[..., :r]
    pairs = head.unflatten(-1, (r // 2, 2)) if s["interleaved"] else head.unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(pairs[..., 0].contiguous(), pairs[..., 1].contiguous()) * f)
    z = z if s["interleaved"] else z.transpose(-1, -2)
    return torch.cat([z.flatten(-2), x[..., r:]], -1)


def _exact_append(s):
    h, d, ps = s["kv_heads"], s["dim"], s["page"]
    keys, values = s["k_cache"].double(), s["v_cache"].double()
    start, lens = s["start"].tolist(), s["kv_len"].tolist()
    queries = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, total in enumerate(lens):
        rows = slice(start[b], start[b + 1])
        n = start[b + 1] - start[b]
        pos = torch.arange(total - n, total, device=DEV)
        page, slot = s["table"][b][pos // ps].long(), pos % ps
        queries[rows] = _exact_turn(s, s["q"][rows].double().view(n, -1, d), pos).reshape(n, -1)
        k = _exact_turn(s, s["k"][rows].double().view(n, h, d), pos)
        for c in range(_chunks(d)):
            part = k[:, :, 8 * c:8 * c + 8]
            keys[page, :, c, slot, :part.shape[2]] = part
        values.transpose(3, 4)[page, :, slot // 8, slot % 8] = s["v"][rows].double().view(n, h, d)
    return [queries, keys, values]


def _exact_shared(s):
    """Sequence by sequence over all of its tokens, the prefix from its group's first row."""
    h, d, ps = s["kv_heads"], s["dim"], s["page"]
    g = s["heads"] // h
    out = torch.zeros(s["q"].shape[0], s["heads"], d, dtype=torch.float64, device=DEV)
    q = s["q"].double().view(-1, s["heads"], d)
    for i, prefix in enumerate(s["prefixes"]):
        for b in range(s["starts"][i], s["starts"][i + 1]):
            total = s["lens"][b]
            pos = torch.arange(total, device=DEV)
            row = torch.where(pos < prefix, s["starts"][i], b)
            page, slot = s["table"][row, pos // ps].long(), pos % ps
            seen = (pos >= total - s["window"]) | (pos < s["sinks"]) if s["window"] else pos >= 0
            for head in range(h):
                k = s["k_cache"][page, head, :, slot].double().flatten(1)[:, :d]
                v = s["v_cache"][page, head, slot // 8, :, slot % 8].double()
                x = (q[b, head * g:(head + 1) * g] @ k.t() * s["scale"]).masked_fill(~seen, -math.inf)
                out[b, head * g:(head + 1) * g] = torch.softmax(x, -1) @ v
    return out.view(s["q"].shape[0], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm":
        return _exact_norm(s)
    if case["kind"] == "rope":
        return _exact_turn(s, s["in"].double().view(case["tokens"], case["heads"], case["dim"]), s["pos"]).reshape(s["in"].shape)
    return _exact_append(s) if case["kind"] == "append" else _exact_shared(s)
