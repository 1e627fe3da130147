"""The token mixers of a hybrid model's layers on its pages and state slots, as measurable cases.

A case is one pass of one layer: new tokens' queries and keys normed and rotated, the keys and values put into the
paged cache; the bounds of pages' keys; a long cache's pages chosen for each query by those bounds and attended over;
or the gated delta rule of a recurrent layer, for prompts, drafts or one token of every sequence.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"bf16": 2, "fp16": 2, "e4m3": 1}
_ctx = None


def _library():
    from paper_2609_15021_gb300 import kvxfer
    return kvxfer


def _context():
    """The one context that a program makes at start-up and keeps."""
    global _ctx
    if _ctx is None:
        _ctx = _library().KvTransfer(0)
    return _ctx.ctx


# ---------------------------------------------------------------- cases


def _rotary(name, seqs, tokens, before, kv_heads, q_heads, head_dim, rotary_dim, block, layout, type, cache, per_block=1,
            interleaved=False, norm=True, moved=False):
    """tokens: of all prompts together, 0 for one token of every sequence; before: the longest context in front of one;
    moved: positions are given, as they are not the cache's after an eviction."""
    return {"name": name, "op": "rotary", "seqs": seqs, "tokens": tokens, "before": before, "kv_heads": kv_heads,
            "q_heads": q_heads, "head_dim": head_dim, "rotary_dim": rotary_dim, "block": block, "layout": layout,
            "type": type, "cache": cache, "per_block": per_block, "interleaved": interleaved, "norm": norm,
            "moved": moved}


def _bounds(name, seqs, shortest, longest, kv_heads, head_dim, block, layout, cache, per_block=1):
    return {"name": name, "op": "bounds", "seqs": seqs, "shortest": shortest, "longest": longest, "kv_heads": kv_heads,
            "head_dim": head_dim, "block": block, "layout": layout, "cache": cache, "per_block": per_block}


def _sparse(name, seqs, shortest, longest, kv_heads, q_heads, head_dim, block, layout, type, cache, budget, sinks=1,
            recent=2, new=1, per_block=1, softcap=0.0, idle=0):
    """Lengths are spread from shortest to longest over their logarithm; budget, sinks and recent are pages; idle:
    sequences of length 0, as the unused places of a batch of fixed size are."""
    return {"name": name, "op": "sparse", "seqs": seqs, "shortest": shortest, "longest": longest, "kv_heads": kv_heads,
            "q_heads": q_heads, "head_dim": head_dim, "block": block, "layout": layout, "type": type, "cache": cache,
            "budget": budget, "sinks": sinks, "recent": recent, "new": new, "per_block": per_block,
            "softcap": softcap, "idle": idle}


def _delta(name, seqs, tokens, heads, head_dim, state_dim, groups, type, fresh=False):
    """tokens: of all prompts together, 0 for one token of every sequence."""
    return {"name": name, "op": "delta", "seqs": seqs, "tokens": tokens, "heads": heads, "head_dim": head_dim,
            "state_dim": state_dim, "groups": groups, "type": type, "fresh": fresh}


def listed():
    return [
        # One user's next token on the 27B-class attention shape (8 KV heads x 128): launch and latency.
        _rotary("rotary_token", 1, 0, 1793, 8, 32, 128, 128, 16, "hnd", "bf16", "bf16"),
        # The next tokens of a serving batch of 48 sequences, NHD pages, rows of 96 elements of which 48 are rotated in
        # neighbouring pairs, no norms.
        _rotary("rotary_batch", 48, 0, 16384, 8, 16, 96, 48, 16, "nhd", "fp16", "fp16", interleaved=True, norm=False),
        # New turns' prompts on the paper's FP8 shape (4 KV heads x 256, a quarter of them rotated) behind contexts that an
        # eviction shrank, so that positions run ahead of the cache's.
        _rotary("rotary_prompt_fp8", 5, 16384, 30000, 4, 24, 256, 64, 32, "hnd", "bf16", "e4m3", per_block=49, moved=True),
        # The bounds of two long documents' pages, made once after they were restored.
        _bounds("bounds_restored", 2, 21003, 32768, 8, 128, 16, "hnd", "bf16"),
        # One user's next token over a 32k document, 64 of whose 2,048 pages are read.
        _sparse("sparse_reply", 1, 32768, 32768, 8, 32, 128, 16, "hnd", "bf16", "bf16", 64),
        # A serving batch of 48 places, 3 of them idle, contexts from one token to 16k, NHD pages, capped scores.
        _sparse("sparse_ragged", 48, 1, 16384, 8, 16, 96, 16, "nhd", "fp16", "fp16", 48, softcap=30.0, idle=3),
        # The paper's FP8 shape at its 127,008-token context, four draft tokens verified at once: 128 of some 4,000 pages.
        _sparse("sparse_fp8_128k", 4, 98765, 127008, 4, 24, 256, 32, "hnd", "bf16", "e4m3", 128, new=4, per_block=49),
        # One user's next token through the hybrid shape's recurrent state (16 heads of 128 x 128): latency.
        _delta("delta_reply", 1, 0, 16, 128, 128, 8, "bf16"),
        # One token of 96 sequences: the states are read and written once.
        _delta("delta_token", 96, 0, 16, 128, 128, 8, "bf16"),
        # Drafts of 16 sequences, some of few tokens, verified at once.
        _delta("delta_draft", 16, 67, 16, 128, 128, 8, "bf16"),
        # The new turn of the hybrid session, 2,048 tokens on a restored state.
        _delta("delta_turn", 1, 2048, 16, 128, 128, 8, "bf16"),
        # Prompts of six sequences from one token to over ten thousand, 24k tokens in all: the largest.
        _delta("delta_prompts", 6, 24001, 16, 128, 128, 16, "fp16", fresh=True),
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotary"] * 3 + ["bounds"] + ["sparse"] * 4 + ["delta"] * 4)
    type = rng.choice(["bf16", "fp16"])
    cache = rng.choice([type, type, "e4m3"])
    head_dim = rng.choice([64, 96, 128, 256] if cache == "e4m3" else [64, 96, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    block = rng.choice([16, 32])
    layout = rng.choice(["hnd", "nhd"])
    per_block = 49 if cache == "e4m3" and rng.random() < 0.5 else 1
    if op == "rotary":
        seqs = _between(rng, 1, 64)
        tokens = rng.choice([0, _between(rng, max(seqs, 2), 16384)])
        return _rotary("", seqs, tokens, _between(rng, 1, 30000), kv_heads, kv_heads * rng.choice([1, 2, 4, 6]), head_dim,
                       rng.choice([head_dim, head_dim // 2, head_dim // 4]), block, layout, type, cache, per_block,
                       interleaved=rng.random() < 0.4, norm=rng.random() < 0.7, moved=rng.random() < 0.3)
    if op == "bounds":
        longest = _between(rng, 1, 32768)
        return _bounds("", rng.randint(1, 3), _between(rng, 1, longest), longest, kv_heads, head_dim, block, layout, cache,
                       per_block)
    if op == "sparse":
        longest = _between(rng, 1, 127008)
        seqs = _between(rng, 1, max(1, min(64, 300000 // longest)))
        budget = _between(rng, 4, 256)
        return _sparse("", seqs, _between(rng, 1, longest), longest, kv_heads, kv_heads * rng.choice([1, 2, 4, 6, 8]),
                       head_dim, block, layout, type, cache, budget, sinks=rng.randint(0, 2), recent=rng.randint(1, 2),
                       new=rng.choice([1, 1, 1, 2, 4]), per_block=per_block, softcap=rng.choice([0.0, 0.0, 30.0]),
                       idle=rng.choice([0, 0, seqs // 8]))
    seqs = _between(rng, 1, 96)
    tokens = rng.choice([0, _between(rng, 2, 24001), _between(rng, 2, 24001)])
    if tokens:
        seqs = min(seqs, 8 if tokens > 2000 else 16, tokens)
    return _delta("", seqs, tokens, rng.choice([8, 16]), rng.choice([64, 128]), rng.choice([64, 128]),
                  rng.choice([2, 4, 8]), type, fresh=rng.random() < 0.5)


# ---------------------------------------------------------------- inputs


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _spread(n, lo, hi, seed=1):
    """n lengths from lo to hi, evenly over the logarithm, the longest first, the others in no order.  A case's
    lengths are the same for every seed of its inputs."""
    if n == 1:
        return [hi]
    got = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * i / (n - 1)))) for i in range(n)]
    order = torch.randperm(n - 1, generator=torch.Generator().manual_seed(seed)).tolist()
    return [got[-1]] + [got[i] for i in order]


def _shares(n, total, seed=1):
    """total cut into n parts of at least one, of quite different sizes, in no order."""
    w = [4.0 ** -i for i in range(n)]
    got = [1 + int((total - n) * x / sum(w)) for x in w]
    got[0] += total - sum(got)
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed)).tolist()
    return [got[i] for i in order]


def _normal(shape, dtype, g, scale=1.0):
    """Normal numbers; a cache's, which are gigabytes, in one draw per 2^28."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        part = flat[a:a + (1 << 28)]
        part.copy_(torch.randn(part.numel(), generator=g, device="cuda") * scale)
    return out


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _pages(case, tokens, g):
    """(one layer's pages, block tables in a random order of the pages)."""
    span = case["block"] * case["per_block"]
    need = [-(-n // span) for n in tokens]
    blocks = sum(need) + 2
    order = torch.randperm(blocks, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((len(tokens), max(need) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = order[at:at + n]
        at += n
    h, b, d = case["kv_heads"], case["block"], case["head_dim"]
    page = (2, h, b, d) if case["layout"] == "hnd" else (2, b, h, d)
    return _normal((blocks * case["per_block"],) + page, _TYPES[case["cache"]], g), tables


def _scales(case):
    return (0.75, 1.25) if case["cache"] == "e4m3" else (1.0, 1.0)


def _pool(case, pages):
    k = _library()
    return k.KvPool.from_tensors([pages], case["kv_heads"], case["block"],
                                 k.KVX_LAYOUT_HND if case["layout"] == "hnd" else k.KVX_LAYOUT_NHD, case["per_block"])


def _new_tokens(case):
    s = case["seqs"]
    return _shares(s, max(case["tokens"], s)) if case["tokens"] else [1] * s


def _prepare_rotary(case, seed):
    g = _generator(seed)
    s, h, hq, d, r = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"], case["rotary_dim"]
    new = _new_tokens(case)
    before = _spread(s, 1, case["before"], 2)
    lengths = [a + b for a, b in zip(new, before)]
    pages, tables = _pages(case, lengths, g)
    starts = [sum(new[:i]) for i in range(s + 1)]
    dtype = _TYPES[case["type"]]
    # one projection's output holds the new tokens' queries, keys and values side by side
    qkv = _normal((starts[-1], hq + 2 * h, d), dtype, g, 2.0)
    st = {"case": case, "pages": pages, "tables": tables, "lengths": _ints(lengths), "starts": _ints(starts),
          "q": qkv[:, :hq], "k": qkv[:, hq:hq + h], "v": qkv[:, hq + h:],
          "out": torch.empty((starts[-1], hq, d), dtype=dtype, device="cuda"),
          "inv_freq": (10000.0 ** (-2.0 * torch.arange(r // 2, device="cuda", dtype=torch.float64) / r)).float(),
          "q_weight": _normal((d,), dtype, g, 0.1) + 1 if case["norm"] else None,
          "k_weight": _normal((d,), dtype, g, 0.1) + 1 if case["norm"] else None, "positions": None}
    if case["moved"]:
        seq = torch.repeat_interleave(torch.arange(s, device="cuda"), _ints(new))
        at = st["lengths"][seq] - (st["starts"][seq + 1] - torch.arange(starts[-1], device="cuda"))
        st["positions"] = (at + 3 * st["lengths"][seq]).to(torch.int32)
    if own:
        k = _library()
        st["pool"] = _pool(case, pages)
        st["batch"] = k.KvBatch(tables, st["lengths"], max_length=max(lengths))
        st["rotary"] = k.KvRotary(hq, st["inv_freq"], interleaved=case["interleaved"], q_weight=st["q_weight"],
                                  k_weight=st["k_weight"], eps=1e-6)
    return st


def _lengths(case):
    got = _spread(case["seqs"], case["shortest"], case["longest"])
    for i in range(min(case.get("idle", 0), case["seqs"] - 1)):
        got[-1 - i] = 0
    return got


def _room_for_bounds(case, pages):
    shape = (pages.shape[0], case["kv_heads"])
    return (torch.zeros(shape + (2, case["head_dim"]), dtype=torch.int8, device="cuda"),
            torch.zeros(shape, dtype=torch.float32, device="cuda"))


def _prepare_bounds(case, seed):
    g = _generator(seed)
    lengths = _lengths(case)
    pages, tables = _pages(case, lengths, g)
    boxes, sizes = _room_for_bounds(case, pages)
    st = {"case": case, "pages": pages, "tables": tables, "lengths": _ints(lengths), "longest": max(lengths),
          "boxes": boxes, "sizes": sizes}
    if own:
        k = _library()
        st["pool"] = _pool(case, pages)
        st["batch"] = k.KvBatch(tables, st["lengths"], max_length=max(lengths))
        st["bounds"] = k.KvBounds(boxes, sizes)
    return st


def _prepare_sparse(case, seed):
    g = _generator(seed)
    lengths = _lengths(case)
    pages, tables = _pages(case, lengths, g)
    s, t, h, hq, d = case["seqs"], case["new"], case["kv_heads"], case["q_heads"], case["head_dim"]
    boxes, sizes = _room_for_bounds(case, pages)
    dtype = _TYPES[case["type"]]
    qkv = _normal((s * t, hq + 2 * h, d), dtype, g)
    qkv[:, :hq] *= 1.5
    st = {"case": case, "pages": pages, "tables": tables, "lengths": _ints(lengths), "longest": max(lengths),
          "boxes": boxes, "sizes": sizes, "q": qkv[:, :hq],
          "selected": torch.empty((s * t, h, case["budget"]), dtype=torch.int32, device="cuda"),
          "out": torch.empty((s * t, hq, d), dtype=dtype, device="cuda"),
          "lse": torch.empty((s * t, hq), dtype=torch.float32, device="cuda")}
    _bounds_of(st, torch.zeros_like(st["lengths"]))  # of all pages: what earlier steps left
    if own:
        k = _library()
        ks, vs = _scales(case)
        st["pool"] = _pool(case, pages)
        st["batch"] = k.KvBatch(tables, st["lengths"], max_length=max(lengths))
        st["bounds"] = k.KvBounds(boxes, sizes)
        st["selection"] = k.KvSelection(hq, case["budget"], sinks=case["sinks"], recent=case["recent"], new_tokens=t)
        st["attention"] = k.KvAttention(hq, new_tokens=t, softcap=case["softcap"], k_scale=ks, v_scale=vs)
        st["select_space"] = k.kv_select_workspace(_context(), st["pool"], st["batch"], st["selection"])
        st["attend_space"] = k.kv_attend_selected_workspace(_context(), st["pool"], st["batch"], st["attention"],
                                                            case["budget"])
    return st


def _prepare_delta(case, seed):
    g = _generator(seed)
    s, h, p, n, gr = case["seqs"], case["heads"], case["head_dim"], case["state_dim"], case["groups"]
    dtype = _TYPES[case["type"]]
    lens = _new_tokens(case)
    size = h * p * n * 4
    slot_bytes = -(-(size + 4096) // 4096) * 4096
    # the slots that are read lie in the first half, the ones written in the second
    pool = torch.zeros(2 * s, slot_bytes, dtype=torch.uint8, device="cuda")
    at = torch.randperm(s, generator=g, device="cuda").to(torch.int32)
    to = torch.randperm(s, generator=g, device="cuda").to(torch.int32) + s
    inner = pool[:, :size].view(torch.float32).view(2 * s, h, p, n)
    inner.copy_(_normal(inner.shape, torch.float32, g, 0.5))
    starts = [sum(lens[:i]) for i in range(s + 1)]
    t = starts[-1]
    # the convolution's output holds queries, keys and values side by side, all of them past a SiLU, so that keys of a
    # sequence have much in common
    wide = torch.nn.functional.silu(_normal((t, 2 * gr * n + h * p), torch.float32, g, 1.5)).to(dtype)
    gates = _normal((t, 2 * h), dtype, g)
    step = torch.exp(torch.rand(h, generator=g, device="cuda") * math.log(100.0) + math.log(1e-3))
    st = {"case": case, "pool": pool, "state": inner, "from": at, "to": to, "starts": _ints(starts), "lens": lens,
          "q": wide[:, :gr * n].view(t, gr, n), "k": wide[:, gr * n:2 * gr * n].view(t, gr, n),
          "v": wide[:, 2 * gr * n:].view(t, h, p), "dt": gates[:, :h], "beta": gates[:, h:],
          "A": -(1.0 + 15.0 * torch.rand(h, generator=g, device="cuda")),
          "dt_bias": torch.log(torch.expm1(step)), "out": torch.empty((t, h, p), dtype=dtype, device="cuda"),
          # a sequence that begins here has no state yet, whatever its slot holds
          "fresh": _ints([int(case["fresh"] and i % 2 == 0) for i in range(s)])}
    if own:
        k = _library()
        st["slots"] = k.StateSlots(pool, 2 * s, slot_bytes, recurrent_offset=0, conv_offset=size)
        st["state_batch"] = k.StateBatch(at, to, starts=st["starts"] if case["tokens"] else None, tokens=t,
                                         fresh=st["fresh"])
        st["workspace"] = k.kv_state_delta_workspace(_context(), st["state_batch"], h, p, n)
    return st


def prepare(case, seed):
    return globals()["_prepare_" + case["op"]](case, seed)


# ---------------------------------------------------------------- plain forms


def _place(st, seq, pos):
    """(page, token of the page) of positions `pos` of sequences `seq` (of one shape)."""
    c = st["case"]
    block = (pos // (c["block"] * c["per_block"])).clamp(0, st["tables"].shape[1] - 1)
    entry = st["tables"][seq, block].long().clamp(min=0)
    return entry * c["per_block"] + (pos // c["block"]) % c["per_block"], pos % c["block"]


def _raw(pages):
    """The pages as elements that can be gathered and scattered, whatever their type."""
    return pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages


def _rows_at(st):
    """(sequence, position in its cache) of every new row."""
    starts = st["starts"].long()
    row = torch.arange(st["q"].shape[0], device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    return seq, st["lengths"].long()[seq] - (starts[seq + 1] - row)


def _normed(x, weight):
    x = x.float()
    return x if weight is None else x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()


def _rotated(st, x, cos, sin):
    r = st["case"]["rotary_dim"]
    part = x[..., :r]
    if st["case"]["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = part[..., :r // 2], part[..., r // 2:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _rotary_plain(st):
    c = st["case"]
    seq, at = _rows_at(st)
    pos = at if st["positions"] is None else st["positions"]
    angle = pos.double()[:, None, None] * st["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    st["out"].copy_(_rotated(st, _normed(st["q"], st["q_weight"]), cos, sin))
    rows = torch.stack([_rotated(st, _normed(st["k"], st["k_weight"]), cos, sin), st["v"].float()], 1)
    if c["cache"] == "e4m3":
        scale = torch.tensor(_scales(c), device="cuda").view(1, 2, 1, 1)
        rows = (rows / scale).clamp(-448.0, 448.0)
    page, slot = _place(st, seq, at)
    rows = _raw(rows.to(st["pages"].dtype))
    if c["layout"] == "hnd":
        _raw(st["pages"])[page, :, :, slot] = rows
    else:
        _raw(st["pages"])[page, :, slot] = rows
    return _rotary_outputs(st)


def _rotary_outputs(st):
    return {"out": st["out"], "pages": st["pages"]}


def _most():
    """127 as a tensor: divided by, where a number would be multiplied by its reciprocal."""
    return torch.full((), 127.0, device="cuda")


def _keys_of(st, page):
    """Keys [..][head][token][element] of pages `page` [..], in 32 bits."""
    c = st["case"]
    got = _raw(st["pages"])[:, 0][page].view(st["pages"].dtype).float()
    return got if c["layout"] == "hnd" else got.transpose(-3, -2)


def _bounds_of(st, first):
    """The bounds of the pages that hold tokens first[s] .. lengths[s] - 1 of every sequence."""
    c = st["case"]
    b = c["block"]
    lengths, first = st["lengths"].long(), first.long()
    index = torch.arange(-(-st["longest"] // b), device="cuda").expand(c["seqs"], -1)
    there = (index * b < lengths[:, None]) & ((index + 1) * b > first[:, None])
    seq, index = torch.nonzero(there, as_tuple=True)[0], index[there]
    page, _ = _place(st, seq, index * b)
    keys = _keys_of(st, page)
    held = (index[:, None] * b + torch.arange(b, device="cuda") < lengths[seq, None])[:, None, :, None]
    low = torch.where(held, keys, math.inf).amin(-2)
    high = torch.where(held, keys, -math.inf).amax(-2)
    size = torch.maximum(low.abs(), high.abs()).amax(-1) / _most()
    by = torch.where(size > 0, size, 1.0)[..., None]
    st["boxes"][page] = torch.stack([(low / by).floor(), (high / by).ceil()], 2).clamp(-127, 127).to(torch.int8)
    st["sizes"][page] = size


def _bounds_plain(st):
    _bounds_of(st, torch.zeros_like(st["lengths"]))
    return _bounds_outputs(st)


def _bounds_outputs(st):
    return {"boxes": st["boxes"], "sizes": st["sizes"]}


def _select_plain(st):
    c = st["case"]
    s, t, h, hq, d, b, budget = (c[x] for x in ("seqs", "new", "kv_heads", "q_heads", "head_dim", "block", "budget"))
    n = -(-st["longest"] // b)
    q = st["q"].float()
    step = q.abs().amax(-1, keepdim=True) / _most()
    whole = torch.round(q / torch.where(step > 0, step, 1.0)).view(s, t, h, hq // h, d).permute(0, 2, 1, 3, 4)
    index = torch.arange(n, device="cuda")
    seq = torch.arange(s, device="cuda")[:, None].expand(s, n)
    page, _ = _place(st, seq, (index * b).expand(s, n))
    box = st["boxes"][page].float().permute(0, 2, 3, 1, 4)  # [s][h][2][n][d]
    rows = whole.reshape(s, h, t * (hq // h), d)
    dot = rows.clamp(min=0) @ box[:, :, 1].transpose(-1, -2) + rows.clamp(max=0) @ box[:, :, 0].transpose(-1, -2)
    dot = dot.view(s, h, t, hq // h, n) * step.view(s, t, h, hq // h, 1).transpose(1, 2)
    score = dot.amax(3) * st["sizes"][page].transpose(1, 2)[:, :, None]  # [s][h][t][n]
    at = st["lengths"].long()[:, None] - t + torch.arange(t, device="cuda")
    pages = torch.where(at >= 0, at // b + 1, 0)[:, None, :, None]  # that the query sees
    forced = (index < c["sinks"]) | (index >= pages - c["recent"])
    rank = (index < pages).long() + ((index < pages) & forced).long()
    order = torch.sort(score, dim=-1, descending=True, stable=True)[1]
    ranked = torch.gather(rank.expand_as(order), -1, order)
    order = torch.gather(order, -1, torch.sort(ranked, dim=-1, descending=True, stable=True)[1])
    wide = torch.full((s, h, t, budget), n, dtype=torch.long, device="cuda")
    m = min(budget, n)
    wide[..., :m] = order[..., :m]
    gone = torch.arange(budget, device="cuda") >= pages.clamp(max=budget)
    picked = torch.sort(wide.masked_fill(gone, n), -1)[0].masked_fill(gone, -1)
    st["selected"].view(s, t, h, budget).copy_(picked.transpose(1, 2))


def _sparse_plain(st):
    c = st["case"]
    s, t, h, hq, d, b, budget = (c[x] for x in ("seqs", "new", "kv_heads", "q_heads", "head_dim", "block", "budget"))
    _bounds_of(st, (st["lengths"] - t).clamp(min=0))
    _select_plain(st)
    picked = st["selected"].long()  # [s * t][h][budget]
    seq = torch.arange(s, device="cuda").repeat_interleave(t)[:, None, None].expand_as(picked)
    page, _ = _place(st, seq, picked.clamp(min=0) * b)
    head = torch.arange(h, device="cuda")[:, None].expand_as(picked)
    raw = _raw(st["pages"])
    got = raw[page, :, head] if c["layout"] == "hnd" else raw[page, :, :, head]  # [..][2][b][d]
    key, value = got.view(st["pages"].dtype).float().movedim(3, 0).reshape(2, s * t, h, budget * b, d)
    ks, vs = _scales(c)
    q = st["q"].float().view(s * t, h, hq // h, d)
    score = (q @ key.transpose(-1, -2)) * (ks / math.sqrt(d))
    if c["softcap"]:
        score = c["softcap"] * torch.tanh(score / c["softcap"])
    at = (st["lengths"].long()[:, None] - t + torch.arange(t, device="cuda")).flatten()
    pos = (picked[..., None] * b + torch.arange(b, device="cuda")).flatten(2)
    seen = (picked >= 0).repeat_interleave(b, -1) & (pos <= at[:, None, None])
    score = score.masked_fill(~seen[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    value = value.masked_fill(~seen[..., None], 0.0)
    st["out"].copy_(((p / total.clamp(min=1e-30)) @ value * vs).view(s * t, hq, d))
    st["lse"].copy_((torch.log(total) + top).view(s * t, hq))
    return _sparse_outputs(st)


def _sparse_outputs(st):
    return {"out": st["out"], "lse": st["lse"], "selected": st["selected"], "boxes": st["boxes"], "sizes": st["sizes"]}


def _delta_plain(st):
    """Chunks of 64 tokens: what the tokens of a chunk write follows from a triangular system, and the chunks from one
    another."""
    c = st["case"]
    s, h, p, n, gr, most = c["seqs"], c["heads"], c["head_dim"], c["state_dim"], c["groups"], max(st["lens"])
    q = min(64, most)
    chunks = -(-most // q)
    starts = st["starts"].long()
    row = torch.arange(st["v"].shape[0], device="cuda")
    seq = torch.searchsorted(starts, row, right=True) - 1
    at = row - starts[seq]

    def spread(v):  # [sequence][chunk][head][token of the chunk][..], zeros behind the last
        wide = torch.zeros((s, chunks * q) + v.shape[1:], device="cuda")
        wide[seq, at] = v.float()
        return wide.view((s, chunks, q) + v.shape[1:]).transpose(2, 3)

    def unit(v):
        v = v.float()
        return (v * torch.rsqrt((v * v).sum(-1, keepdim=True) + 1e-6)).repeat_interleave(h // gr, 1)

    raw = st["dt"].float() + st["dt_bias"]
    step = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))
    beta = spread(1 / (1 + torch.exp(-st["beta"].float())))[..., None]
    decay = torch.cumsum(spread(step * st["A"]).double(), -1)  # of the state up to a token, as a logarithm
    key, query, value = spread(unit(st["k"])), spread(unit(st["q"])) / math.sqrt(n), spread(st["v"])
    below = torch.ones((q, q), dtype=torch.bool, device="cuda").tril()
    pair = torch.exp((decay[..., :, None] - decay[..., None, :]).float().masked_fill(~below, -math.inf))
    last, decay = torch.exp((decay[..., -1:] - decay).float())[..., None], torch.exp(decay.float())[..., None]
    system = (key @ key.transpose(-1, -2) * pair * beta).tril(-1)
    solved = torch.eye(q, device="cuda").expand_as(system).clone()
    for i in range(1, q):
        solved[..., i, :] -= (system[..., i:i + 1, :i] @ solved[..., :i, :])[..., 0, :]
    writes, reads = solved @ (value * beta), solved @ (key * (beta * decay))
    inner, query, key = query @ key.transpose(-1, -2) * pair, query * decay, key * last
    state = st["state"][st["from"].long()] * (st["fresh"] == 0).view(s, 1, 1, 1)  # [s][h][p][n]
    y = torch.empty_like(value)
    for i in range(chunks):
        new = writes[:, i] - reads[:, i] @ state.transpose(-1, -2)
        y[:, i] = query[:, i] @ state.transpose(-1, -2) + inner[:, i] @ new
        state = state * decay[:, i, :, -1:] + new.transpose(-1, -2) @ key[:, i]
    st["out"].copy_(y.transpose(2, 3).reshape(s, chunks * q, h, p)[seq, at])
    st["state"][st["to"].long()] = state
    return _delta_outputs(st)


def _delta_outputs(st):
    return {"out": st["out"], "state": st["state"][st["case"]["seqs"]:]}


# ---------------------------------------------------------------- the framework's operators


def _rotary_own(st):
    ks, vs = _scales(st["case"])
    _library().kv_append_rotary(_context(), st["pool"], 0, st["batch"], st["rotary"], st["q"], st["k"], st["v"], st["out"],
                                positions=st["positions"], starts=st["starts"] if st["case"]["tokens"] else None,
                                k_scale=ks, v_scale=vs)
    return _rotary_outputs(st)


def _bounds_own(st):
    _library().kv_bounds(_context(), st["pool"], 0, st["batch"], st["bounds"], new_tokens=st["longest"])
    return _bounds_outputs(st)


def _sparse_own(st):
    k, ctx = _library(), _context()
    k.kv_bounds(ctx, st["pool"], 0, st["batch"], st["bounds"], new_tokens=st["case"]["new"])
    k.kv_select(ctx, st["pool"], st["batch"], st["bounds"], st["selection"], st["q"], st["selected"], st["select_space"])
    k.kv_attend_selected(ctx, st["pool"], 0, st["batch"], st["attention"], st["selected"], st["q"], st["out"],
                         st["attend_space"], lse=st["lse"])
    return _sparse_outputs(st)


def _delta_own(st):
    _library().kv_state_delta(_context(), st["slots"], st["state_batch"], st["q"], st["k"], st["v"], st["beta"], st["out"],
                              dt=st["dt"], A=st["A"], dt_bias=st["dt_bias"], workspace=st["workspace"])
    return _delta_outputs(st)


def run(state):
    return globals()["_%s_%s" % (state["case"]["op"], "own" if own else "plain")](state)


# ---------------------------------------------------------------- what a pass cannot do without


def work(case):
    c, op = case, case["op"]
    if op == "rotary":
        tokens = sum(_new_tokens(c))
        row, size = c["kv_heads"] * c["head_dim"], _SIZE[c["type"]]
        return {"bytes": tokens * (2 * c["q_heads"] * c["head_dim"] * size + 2 * row * (size + _SIZE[c["cache"]])),
                "flops": tokens * (c["q_heads"] + c["kv_heads"]) * (3 * c["rotary_dim"] + 4 * c["head_dim"])}
    if op == "bounds":
        pages = sum(-(-x // c["block"]) for x in _lengths(c))
        row = c["kv_heads"] * c["head_dim"]
        return {"bytes": sum(_lengths(c)) * row * _SIZE[c["cache"]] + pages * (2 * row + 4 * c["kv_heads"]), "flops": 0}
    if op == "sparse":
        h, d, b, group = c["kv_heads"], c["head_dim"], c["block"], c["q_heads"] // c["kv_heads"]
        size = _SIZE[c["cache"]]
        got = flops = 0
        for x in _lengths(c):
            pages = -(-x // b)
            # the bounds are scored once for all new tokens; the pages that are read are each query's own
            picked = sum(min(c["budget"], -(-max(0, x - i) // b)) for i in range(c["new"]))
            got += h * (pages * (2 * d + 4) + picked * (2 * b * d * size + 4))
            flops += h * group * (4 * c["new"] * pages * d + 4 * picked * b * d)
        tokens = c["seqs"] * c["new"]
        return {"bytes": got + tokens * c["q_heads"] * (2 * d * _SIZE[c["type"]] + 4), "flops": flops}
    tokens = sum(_new_tokens(c))
    h, p, n = c["heads"], c["head_dim"], c["state_dim"]
    rows = tokens * (2 * h * p + 2 * c["groups"] * n + 2 * h) * _SIZE[c["type"]]
    # the recurrence itself: decay, what the state holds for the key, update and read-out of every element of the state
    return {"bytes": rows + 2 * c["seqs"] * h * p * n * 4, "flops": 7 * tokens * h * p * n}


# ---------------------------------------------------------------- the definitions in 64 bits


def _exact_rotary(st):
    """Sequence by sequence; a pair turned as a complex number."""
    c = st["case"]
    r, tables = c["rotary_dim"], st["tables"].tolist()
    lengths, starts = st["lengths"].tolist(), st["starts"].tolist()
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    pages = None if c["cache"] == "e4m3" else st["pages"].double()
    for s in range(c["seqs"]):
        a, b = starts[s], starts[s + 1]
        at = range(lengths[s] - (b - a), lengths[s])
        pos = torch.tensor(list(at), device="cuda") if st["positions"] is None else st["positions"][a:b]
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           pos[:, None].double() * st["inv_freq"].double())[:, None]

        def turned(x, weight):
            x = x.double()
            if weight is not None:
                x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / c["head_dim"] + 1e-6) * weight.double()
            pairs = x[..., :r].unflatten(-1, (r // 2, 2) if c["interleaved"] else (2, r // 2))
            if not c["interleaved"]:
                pairs = pairs.transpose(-1, -2)
            pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            if not c["interleaved"]:
                pairs = pairs.transpose(-1, -2)
            return torch.cat([pairs.flatten(-2), x[..., r:]], -1)

        out[a:b] = turned(st["q"][a:b], st["q_weight"])
        if pages is None:
            continue
        rows = torch.stack([turned(st["k"][a:b], st["k_weight"]), st["v"][a:b].double()], 1)
        page = [tables[s][x // c["block"] // c["per_block"]] * c["per_block"] + x // c["block"] % c["per_block"] for x in at]
        page, slot = torch.tensor(page, device="cuda"), torch.tensor([x % c["block"] for x in at], device="cuda")
        view = pages if c["layout"] == "nhd" else pages.transpose(2, 3)  # [page][2][token][head][d]
        view[page, :, slot] = rows
    return {"out": out, "pages": pages}


def _exact_boxes(st):
    """(pages' boxes, their sizes in 64 bits), sequence by sequence."""
    c = st["case"]
    b, boxes, sizes = c["block"], st["boxes"].clone(), st["sizes"].double()
    for s, length in enumerate(st["lengths"].tolist()):
        n = -(-length // b)
        if n == 0:
            continue
        index = torch.arange(n, device="cuda")
        entry = st["tables"][s, index // c["per_block"]].long()
        page = entry * c["per_block"] + index % c["per_block"]
        keys = st["pages"].view(torch.uint8)[page].view(st["pages"].dtype)[:, 0].double()
        keys = keys.transpose(1, 2) if c["layout"] == "hnd" else keys  # [page][token][head][d]
        low, high = keys.amin(1), keys.amax(1)
        rest = length - (n - 1) * b
        low[-1], high[-1] = keys[-1, :rest].amin(0), keys[-1, :rest].amax(0)
        size = torch.stack([low.abs(), high.abs()]).amax(0).amax(-1) / 127
        sizes[page] = size
        step = size.float().double()[..., None]  # the bounds are whole numbers of the size as it is stored
        ratio = torch.stack([torch.floor((low / step).float()), torch.ceil((high / step).float())], 2)
        boxes[page] = torch.where(step[:, :, None] > 0, ratio, 0.0).clamp(-127, 127).to(torch.int8)
    return boxes, sizes


def _exact_bounds(st):
    return {"boxes": None, "sizes": _exact_boxes(st)[1]}


def _exact_sparse(st):
    """Query by query and head by head: every page's score, the best of them, and attention over their tokens."""
    c = st["case"]
    t, h, hq, d, b = c["new"], c["kv_heads"], c["q_heads"], c["head_dim"], c["block"]
    group, (ks, vs) = hq // h, _scales(c)
    boxes, sizes = _exact_boxes(st)
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    for s, length in enumerate(st["lengths"].tolist()):
        for i in range(t):
            pos = length - t + i
            if pos < 0:
                continue
            n = pos // b + 1
            index = torch.arange(n, device="cuda")
            page = st["tables"][s, index // c["per_block"]].long() * c["per_block"] + index % c["per_block"]
            q = st["q"][s * t + i].double()
            step = (q.abs().amax(-1, keepdim=True) / 127).float().double()
            whole = torch.round((q / step).float()).double()
            always = [x for x in range(n) if x < c["sinks"] or x >= n - c["recent"]]
            for head in range(h):
                low, high = (boxes[page, head, x].double() for x in (0, 1))
                mine = slice(head * group, (head + 1) * group)
                dot = torch.maximum(whole[mine, None] * low, whole[mine, None] * high).sum(-1)
                score = ((dot * step[mine]).float().amax(0).double() * sizes[page, head].float().double()).float()
                score[always] = math.inf
                best = torch.sort(score, descending=True, stable=True)[1][:c["budget"]].sort()[0]
                rows = st["pages"].view(torch.uint8)[page[best]].view(st["pages"].dtype)
                rows = rows[:, :, head] if c["layout"] == "hnd" else rows[:, :, :, head]  # [page][2][token][d]
                rows = rows.double().transpose(0, 1).reshape(2, -1, d)
                seen = ((best * b)[:, None] + torch.arange(b, device="cuda")).flatten() <= pos
                k, v = rows[0, seen] * ks, rows[1, seen] * vs
                logit = q[mine] @ k.T / math.sqrt(d)
                if c["softcap"]:
                    logit = c["softcap"] * torch.tanh(logit / c["softcap"])
                total = torch.logsumexp(logit, -1, keepdim=True)
                out[s * t + i, mine] = torch.exp(logit - total) @ v
                lse[s * t + i, mine] = total[:, 0]
    return {"out": out, "lse": lse, "selected": None, "boxes": None, "sizes": sizes}


def _exact_delta(st):
    """The recurrence, token by token."""
    c = st["case"]
    s, h, gr, n = c["seqs"], c["heads"], c["groups"], c["state_dim"]
    state = st["state"][st["from"].long()].double()
    state[st["fresh"] != 0] = 0
    raw = st["dt"].double() + st["dt_bias"].double()
    alpha = torch.exp(torch.nn.functional.softplus(raw, threshold=1e9) * st["A"].double())
    beta = torch.sigmoid(st["beta"].double())
    unit = [x.double() / torch.sqrt((x.double() ** 2).sum(-1, keepdim=True) + 1e-6) for x in (st["q"], st["k"])]
    starts, longest = st["starts"].long(), max(st["lens"])
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    order = torch.argsort(starts.diff(), descending=True, stable=True)
    lens = sorted(st["lens"], reverse=True)
    state, first = state[order], starts[:-1][order]
    live = s
    for t in range(longest):
        while lens[live - 1] <= t:
            live -= 1
        row = first[:live] + t
        part = state[:live]
        q, k = (x[row].repeat_interleave(h // gr, 1) for x in unit)
        part.mul_(alpha[row][..., None, None])
        wrong = st["v"][row].double() - (part @ k[..., None])[..., 0]
        part.add_((beta[row][..., None] * wrong)[..., None] * k[:, :, None])
        out[row] = (part @ q[..., None])[..., 0] / math.sqrt(n)
    new = torch.zeros(st["state"][s:].shape, dtype=torch.float64, device="cuda")
    new[st["to"].long()[order] - s] = state
    return {"out": out, "state": new}


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    return globals()["_exact_" + case["op"]](state)
