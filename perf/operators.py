"""Cases and plain forms of the serving operators: the paged cache plan, the 8-bit cache write, the
attention that reads the cache, and the linear layer with 4-bit weights.

Each case is one call of one operator.  `run` computes it with elementary torch operations in 32 bits
(`own` false) or with the library's entry points (`own` true); `exact` computes it from its definition
in 64 bits.  Request lengths follow from the case alone (`_lengths`), the seed orders them and fills the data.
"""
import math

import torch

own = False

_FLOAT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_DEV = "cuda"


def listed():
    return [
        # 64 conversations that each add one token: what every step of a decode loop asks first
        {"name": "plan_decode", "op": "plan", "B": 64, "new": 1, "cached": 4096, "page": 16, "ragged": True},
        # 500 prompts admitted at once into an empty cache, a few hundred thousand tokens
        {"name": "plan_prompts", "op": "plan", "B": 500, "new": 2048, "cached": 0, "page": 32, "ragged": True},
        # one new token for each of 64 requests, into pages that are already partly filled
        {"name": "write_decode", "op": "write", "B": 64, "new": 1, "cached": 1000, "heads": 8, "dim": 128, "page": 16,
         "type": "bf16", "ragged": True},
        # prompts of 1 to 4095 tokens that start wherever the page before them ended
        {"name": "write_prompts", "op": "write", "B": 9, "new": 4095, "cached": 333, "heads": 8, "dim": 128, "page": 64,
         "type": "f16", "ragged": True},
        # one user, a short conversation: latency
        {"name": "attn_token_short", "op": "attn", "B": 1, "new": 1, "ctx": 777, "q_heads": 32, "heads": 8, "dim": 128,
         "page": 16, "window": 0, "type": "bf16", "ragged": False},
        # a decode step of a full batch with conversations of every length
        {"name": "attn_batch", "op": "attn", "B": 64, "new": 1, "ctx": 8192, "q_heads": 32, "heads": 8, "dim": 128,
         "page": 16, "window": 0, "type": "f16", "ragged": True},
        # two very long documents being answered
        {"name": "attn_token_long", "op": "attn", "B": 2, "new": 1, "ctx": 131072, "q_heads": 64, "heads": 8, "dim": 128,
         "page": 64, "window": 0, "type": "bf16", "ragged": False},
        # a chunk of a prompt over what the cache holds of it so far
        {"name": "attn_prompt", "op": "attn", "B": 1, "new": 2048, "ctx": 8192, "q_heads": 32, "heads": 8, "dim": 128,
         "page": 32, "window": 0, "type": "bf16", "ragged": False},
        # a layer's smaller projection for one token: latency
        {"name": "w4_token_small", "op": "w4", "M": 1, "N": 4096, "K": 4096, "group": 128, "zero": False, "pad": 32,
         "type": "f16", "out": "f16"},
        # the largest projections for one token: the weights' bytes are the bound
        {"name": "w4_token_large", "op": "w4", "M": 1, "N": 16384, "K": 8192, "group": 64, "zero": True, "pad": 32,
         "type": "bf16", "out": "bf16"},
        # a few tokens, sizes that no tile divides, groups that end inside the last one
        {"name": "w4_ragged", "op": "w4", "M": 7, "N": 5003, "K": 4111, "group": 32, "zero": True, "pad": 32,
         "type": "f16", "out": "f16"},
        # a decode step of a full batch
        {"name": "w4_batch", "op": "w4", "M": 128, "N": 8192, "K": 8192, "group": 128, "zero": False, "pad": 32,
         "type": "bf16", "out": "bf16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["plan", "write", "attn", "attn", "w4", "w4"])
    if op == "plan":
        prompts = rng.random() < 0.5
        B = _log(rng, 1, 500)
        return {"op": op, "B": B, "new": _log(rng, 2, 2048) if prompts else 1,
                "cached": _log(rng, 1, 4096) if rng.random() < 0.7 else 0,
                "page": rng.choice([16, 32, 64, 128]), "ragged": rng.random() < 0.8}
    if op == "write":
        heads, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256])
        new = _log(rng, 1, 4095)
        most = max(1, min(64, 4_000_000 // (new * heads * dim)))
        return {"op": op, "B": _log(rng, 1, most), "new": new, "cached": _log(rng, 1, 1000), "heads": heads, "dim": dim,
                "page": rng.choice([16, 32, 64, 128]), "type": rng.choice(["f16", "bf16"]), "ragged": rng.random() < 0.8}
    if op == "attn":
        heads, dim, ratio = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128, 256]), rng.choice([1, 2, 4, 5, 8])
        kind = {"op": op, "q_heads": heads * ratio, "heads": heads, "dim": dim, "page": rng.choice([16, 32, 64, 128]),
                "type": rng.choice(["f16", "bf16"]), "ragged": rng.random() < 0.7}
        if rng.random() < 0.6:  # single tokens
            ctx = _log(rng, 1, 131072)
            most = max(1, min(64, 2 * 131072 * 8 * 128 // (ctx * heads * dim)))
            return {**kind, "B": _log(rng, 1, most), "new": 1, "ctx": ctx,
                    "window": rng.choice([0, 0, _log(rng, 1, 4096)])}
        pairs = 2048 * 7168 * 32 * 128 // (heads * ratio * dim)
        new = min(_log(rng, 2, 2047), math.isqrt(pairs))
        ctx = min(new + (_log(rng, 1, 6144) if rng.random() < 0.7 else 0), pairs // new)
        most = max(1, min(4, pairs // (new * ctx)))
        return {**kind, "B": _log(rng, 1, most), "new": new, "ctx": ctx, "window": rng.choice([0, 0, _log(rng, 1, 4096)])}
    M = _log(rng, 1, 128)
    return {"op": op, "M": M, "N": _log(rng, 250, 8192), "K": _log(rng, 250, 8192), "group": rng.choice([32, 64, 128, 256]),
            "zero": rng.random() < 0.5, "pad": rng.choice([2, 32, 32]), "type": rng.choice(["f16", "bf16"]),
            "out": rng.choice(["same", "f32"])}


def _lengths(count, most, ragged, least=1):
    """`count` lengths up to `most`: all of them `most`, or spread evenly from `least` to it."""
    if not ragged or count == 1:
        return [most] * count
    return [least + int((most + 1 - least) * (((i + 1) * 0.6180339887498949) % 1.0)) for i in range(count)]


def _requests(case):
    """(cached, new) lengths of each request before the call."""
    B, new = case["B"], _lengths(case["B"], case["new"], case["ragged"])
    if case["op"] == "attn":
        ctx = [max(n, c) for n, c in zip(new, _lengths(B, case["ctx"], case["ragged"]))]
        return [c - n for c, n in zip(ctx, new)], new
    if case["cached"] == 0:
        return [0] * B, new
    return _lengths(B, case["cached"], case["ragged"])[::-1], new


def _group_bytes(case):
    groups = -(-case["K"] // case["group"])
    return case["N"] * groups * (2 + (1 if case["zero"] else 0))


def work(case):
    op = case["op"]
    if op == "w4":
        M, N, K = case["M"], case["N"], case["K"]
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": N * ((K + 1) // 2) + _group_bytes(case) + M * K * 2 + M * N * out, "flops": 2 * M * N * K}
    cached, new = _requests(case)
    page, T = case["page"], sum(new)
    if op == "plan":
        added = sum(-(-(c + n) // page) - -(-c // page) for c, n in zip(cached, new))
        # lengths in; starts, lengths, new table entries (a free page read, an entry written), slots and positions out
        return {"bytes": 4 * (4 * case["B"] + 1) + 8 * added + 12 * T + 16, "flops": 0}
    H, D = case["heads"], case["dim"]
    if op == "write":
        touched = sum((c + n - 1) // page - c // page + 1 for c, n in zip(cached, new))
        # rows and slots in, 8-bit rows and scales out (pages whose scale grows are rewritten besides: not counted)
        return {"bytes": T * (2 * H * D * 3 + 8) + touched * H * 2 * 8, "flops": 4 * T * H * D}
    Hq, window = case["q_heads"], case["window"]
    tokens = pairs = pages = 0
    for c, n in zip(cached, new):
        first = max(0, c + 1 - window) if window else 0
        tokens += c + n - first
        pages += (c + n - 1) // page - first // page + 1
        a, b = c + 1, c + n  # positions see a, a + 1, ..., b tokens, or `window` of them
        if window and a < window:
            cut = min(b, window)
            pairs += (a + cut) * (cut - a + 1) // 2 + window * max(0, b - cut)
        else:
            pairs += window * n if window else (a + b) * n // 2
    return {"bytes": tokens * 2 * H * D + pages * (8 * H + 4) + T * Hq * (4 * D + 4) + 8 * case["B"],
            "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + 13)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEV)


def _codes(g, *shape):
    """8-bit values as a quantised cache holds them: bell-shaped, the largest of a block near 127."""
    x = torch.empty(shape, dtype=torch.float16, device=_DEV).normal_(0.0, 40.0, generator=g)
    return x.round_().clamp_(-127, 127).to(torch.int8)


def _tables(g, cached, new, page, spare):
    """Block tables over a shuffled pool: (table, pages of the pool, pages that no request holds)."""
    have = [-(-c // page) for c in cached]
    want = [-(-(c + n) // page) for c, n in zip(cached, new)]
    width = max(want) + 1
    order = torch.randperm(sum(want) + spare, generator=g, device=_DEV).to(torch.int32)
    hold = torch.tensor(have, device=_DEV)
    start = torch.cumsum(hold, 0) - hold
    col = torch.arange(width, device=_DEV)
    index = (start[:, None] + col).clamp_(max=order.numel() - 1)
    table = torch.where(col < hold[:, None], order[index], -1).to(torch.int32)
    return table, order.numel(), order[sum(have):].contiguous()


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "w4":
        M, N, K, group = case["M"], case["N"], case["K"], case["group"]
        ld = -(-K // case["pad"]) * case["pad"]
        q = torch.empty((N, ld), dtype=torch.float16, device=_DEV).normal_(0.0, 2.7, generator=g)
        q = q.round_().clamp_(-8, 7).to(torch.int8)
        q[:, K:] = 0
        codes = ((q[:, 0::2] & 15) | (q[:, 1::2] << 4)).view(torch.uint8)
        groups = -(-K // group)
        t = _FLOAT[case["type"]]
        scale = (torch.rand((N, groups), generator=g, device=_DEV) * 0.02 + 0.005).to(t)
        zero = torch.randint(-3, 4, (N, groups), generator=g, device=_DEV, dtype=torch.int8) if case["zero"] else None
        x = torch.empty((M, K), dtype=torch.float32, device=_DEV).normal_(generator=g).to(t)
        out = case["type"] if case["out"] == "same" else case["out"]
        return {"op": op, "M": M, "N": N, "K": K, "ld": ld, "group": group, "codes": codes, "scale": scale, "zero": zero, "x": x,
                "type": case["type"], "out": out, "y": torch.empty((M, N), dtype=_FLOAT[out], device=_DEV)}
    cached, new = _requests(case)
    page, B = case["page"], case["B"]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed))).tolist()
    cached, new = [cached[i] for i in order], [new[i] for i in order]
    T = sum(new)
    table, pool, free = _tables(g, cached, new, page, 8)
    s = {"op": op, "B": B, "T": T, "page": page, "cached": _ints(cached), "new": _ints(new), "table": table, "pool": pool,
         "width": table.shape[1]}
    if op == "plan":
        s.update(free=free, slots=torch.empty(T + 5, dtype=torch.int64, device=_DEV), max_tokens=T + 5,
                 positions=torch.empty(T + 5, dtype=torch.int32, device=_DEV),
                 start=torch.empty(B + 1, dtype=torch.int32, device=_DEV), ctx=torch.empty(B, dtype=torch.int32, device=_DEV),
                 counts=torch.empty(4, dtype=torch.int32, device=_DEV))
        return s
    # the pages that the call's own tokens need are in the table by now
    table, _, _ = _tables(g, [c + n for c, n in zip(cached, new)], [0] * B, page, 8)
    H, D, t = case["heads"], case["dim"], _FLOAT[case["type"]]
    start = torch.zeros(B + 1, dtype=torch.int64, device=_DEV)
    start[1:] = torch.cumsum(s["new"], 0)
    s.update(H=H, D=D, type=case["type"], table=table, width=table.shape[1],
             k=_codes(g, pool, H, page, D), v=_codes(g, pool, H, page, D),
             ks=torch.empty((pool, H), device=_DEV).normal_(generator=g).mul_(0.25).exp_().mul_(0.025),
             vs=torch.empty((pool, H), device=_DEV).normal_(generator=g).mul_(0.25).exp_().mul_(0.025),
             start=start.to(torch.int32), ctx=s["cached"] + s["new"])
    if op == "write":
        request = torch.searchsorted(start[1:], torch.arange(T, device=_DEV), right=True)
        pos = s["cached"].long()[request] + torch.arange(T, device=_DEV) - start[request]
        s["slots"] = table[request, pos // page].long() * page + pos % page
        # keys and values are parts of one fused projection, after the queries; some channels are large, as in keys
        wide = torch.empty((T, 6 * H * D), dtype=torch.float32, device=_DEV).normal_(generator=g)
        wide *= torch.empty((1, 6 * H * D), device=_DEV).normal_(generator=g).mul_(0.4).exp_()
        s["rows"] = wide.to(t)
        s["most_pages"] = min(T, T // page + 2 * B)
        return s
    Hq = case["q_heads"]
    s.update(Hq=Hq, window=case["window"], scale=1.0 / math.sqrt(D), most_new=max(new), most_ctx=max(c + n for c, n in zip(cached, new)),
             rows=torch.empty((T, (Hq + 2 * H) * D), dtype=torch.float32, device=_DEV).normal_(generator=g).to(t),
             out=torch.empty((T, Hq, D), dtype=t, device=_DEV), lse=torch.empty((T, Hq), dtype=torch.float32, device=_DEV))
    return s


# ------------------------------------------------------------------ plain forms
def _plain_plan(s):
    page, width, table = s["page"], s["width"], s["table"]
    cached, new = s["cached"].long().clamp(min=0), s["new"].long().clamp(min=0)
    have, want = (cached + page - 1) // page, (cached + new + page - 1) // page
    add = (want.clamp(max=width) - have).clamp(min=0)
    base = torch.cumsum(add, 0) - add
    col = torch.arange(width, device=_DEV)
    index = base[:, None] + col - have[:, None]
    fresh = (col >= have[:, None]) & (col < want[:, None])
    page_of = torch.where(index < s["free"].numel(), s["free"].long()[index.clamp(0, s["free"].numel() - 1)], -1)
    table.copy_(torch.where(fresh, page_of, table.long()))
    start = torch.zeros(s["B"] + 1, dtype=torch.int64, device=_DEV)
    torch.cumsum(new, 0, out=start[1:])
    t = torch.arange(s["max_tokens"], device=_DEV)
    request = torch.searchsorted(start[1:], t, right=True).clamp(max=s["B"] - 1)
    pos = cached[request] + t - start[request]
    held = torch.where(pos // page < width, table[request, (pos // page).clamp(max=width - 1)].long(), -1)
    live = t < start[-1]
    taken = add.sum().clamp(max=s["free"].numel())
    counts = torch.stack([taken, start[-1], (want - have).clamp(min=0).sum() - taken, (cached + new).max()])
    return {"table": table, "slots": torch.where(live & (held >= 0), held * page + pos % page, -1),
            "positions": torch.where(live, pos, -1).to(torch.int32), "start": start.to(torch.int32),
            "ctx": (cached + new).to(torch.int32), "counts": counts.to(torch.int32)}


def _plain_write_one(cache, scale, x, slots, page, most_pages):
    """x: T x H x D.  The scale of a page and head is its largest magnitude over 127 and only grows while the page fills."""
    x = x.float()
    finite = torch.isfinite(x)
    of, at = slots // page, slots % page
    begins = torch.ones_like(of, dtype=torch.bool)
    begins[1:] = of[1:] != of[:-1]
    run = torch.cumsum(begins, 0)  # 1, 2, ...: the tokens of one page stand together
    first = torch.searchsorted(run, torch.minimum(torch.arange(1, most_pages + 1, device=_DEV), run[-1]))
    pages, held = of[first], at[first]  # touched pages (the last one again where there are fewer), tokens already there
    run = run[first][:, None]
    largest = torch.where(finite, x.abs(), 0.0).amax(2)
    most = torch.zeros((of.numel() + 1, x.shape[1]), device=_DEV)
    most.scatter_reduce_(0, torch.cumsum(begins, 0)[:, None].expand_as(largest), largest, "amax")
    most = most[run[:, 0]]
    before = torch.where(held[:, None] > 0, scale[pages], 0.0)
    wanted = torch.where(most < 2.0 ** -100, 0.0, most / 127.0)
    after = torch.maximum(before, wanted)
    grown = after > before
    ratio = torch.where(grown, before / torch.where(grown, after, 1.0), 1.0)
    block = cache[pages]
    keep = torch.arange(page, device=_DEV) < held[:, None]
    again = (block.float() * ratio[:, :, None, None]).round().to(torch.int8)
    cache[pages] = torch.where(keep[:, None, :, None], again, block)
    scale[pages] = after
    s = scale[of]
    inverse = torch.where(s > 0, 1.0 / torch.where(s > 0, s, 1.0), 0.0)[:, :, None]
    y = torch.where(torch.isnan(x), 0.0, torch.where(finite, (torch.where(finite, x, 0.0) * inverse).round(), torch.sign(x) * 127.0))
    cache[of, :, at] = y.clamp(-127, 127).to(torch.int8)


def _plain_write(s):
    H, D, T = s["H"], s["D"], s["T"]
    k, v = s["rows"][:, 4 * H * D:5 * H * D].reshape(T, H, D), s["rows"][:, 5 * H * D:].reshape(T, H, D)
    _plain_write_one(s["k"], s["ks"], k, s["slots"], s["page"], s["most_pages"])
    _plain_write_one(s["v"], s["vs"], v, s["slots"], s["page"], s["most_pages"])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _plain_attn(s):
    B, H, D, Hq, T, page = s["B"], s["H"], s["D"], s["Hq"], s["T"], s["page"]
    G, most = Hq // H, s["most_new"]
    pages = s["table"][:, :-(-s["most_ctx"] // page)].long().clamp(min=0)
    span = pages.shape[1] * page

    def gather(codes, scale):
        x = codes[pages].float().mul_(scale[pages][..., None, None])
        return x.permute(0, 2, 1, 3, 4).reshape(B, H, span, D)

    start, ctx = s["start"].long(), s["ctx"].long()
    n = start[1:] - start[:-1]
    row = torch.arange(most, device=_DEV)
    q = s["rows"][:, :Hq * D].reshape(T, H, G, D)[(start[:-1, None] + row).clamp(max=T - 1)].float()
    q = q.permute(0, 2, 3, 1, 4).reshape(B, H, G * most, D)
    score = (q * s["scale"]) @ gather(s["k"], s["ks"]).transpose(2, 3)
    score = score.view(B, H, G, most, span)
    pos, tok = (ctx - n)[:, None] + row, torch.arange(span, device=_DEV)
    hidden = tok > pos[..., None]
    if s["window"]:
        hidden |= tok <= pos[..., None] - s["window"]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    m = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, G * most, span) @ gather(s["v"], s["vs"])).view(B, H, G, most, D) / total
    o = torch.where(total > 0, o, 0.0)
    lse = torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0]
    request = torch.searchsorted(start[1:], torch.arange(T, device=_DEV), right=True)
    index = torch.arange(T, device=_DEV) - start[request]
    out = o.permute(0, 3, 1, 2, 4)[request, index].reshape(T, Hq, D)
    return {"out": out.to(_FLOAT[s["type"]]), "lse": lse.permute(0, 3, 1, 2)[request, index].reshape(T, Hq)}


def _plain_w4(s):
    c, N, K = s["codes"], s["N"], s["K"]
    w = torch.stack([(c & 15), (c >> 4)], 2).view(N, -1)[:, :K].float()
    w = torch.where(w > 7, w - 16, w)
    group = torch.arange(K, device=_DEV) // s["group"]
    if s["zero"] is not None:
        w = w - s["zero"].float()[:, group]
    w = w * s["scale"].float()[:, group]
    return (s["x"].float() @ w.t()).to(_FLOAT[s["out"]])


# ------------------------------------------------------------------ the library's calls
_lib = {}


def _library():
    if not _lib:
        from paper_2609_24519_b200 import binding
        _lib["b"], _lib["h"] = binding, binding.awe_create(torch.cuda.current_device())
        _lib["type"] = {"f16": binding.F16, "bf16": binding.BF16, "f32": binding.F32}
    return _lib["b"], _lib["h"], _lib["type"]


def _cache(b, s):
    if "cache" not in s:
        s["cache"] = b.kv_cache(s["k"], s["v"], s["ks"], s["vs"], s["pool"], s["H"], s["page"], s["D"])
    return s["cache"]


def _own_plan(s):
    b, h, _ = _library()
    b.awe_kv_plan(h, s["cached"], s["new"], s["B"], s["page"], s["free"], s["free"].numel(), s["table"], s["width"], s["width"],
                  s["slots"], s["positions"], s["max_tokens"], s["start"], s["ctx"], s["counts"])
    return {"table": s["table"], "slots": s["slots"], "positions": s["positions"], "start": s["start"], "ctx": s["ctx"],
            "counts": s["counts"]}


def _own_write(s):
    b, h, types = _library()
    H, D = s["H"], s["D"]
    b.awe_kv_write(h, _cache(b, s), s["rows"][:, 4 * H * D:], s["rows"][:, 5 * H * D:], types[s["type"]], s["T"],
                   6 * H * D, 6 * H * D, s["slots"])
    return {"k": s["k"], "v": s["v"], "ks": s["ks"], "vs": s["vs"]}


def _own_attn(s):
    b, h, types = _library()
    cache, H, D, Hq = _cache(b, s), s["H"], s["D"], s["Hq"]
    if "workspace" not in s:
        s["workspace_bytes"] = b.awe_kv_attention_workspace_bytes(h, cache, s["T"], Hq, s["B"])
        s["workspace"] = torch.empty(max(1, s["workspace_bytes"]), dtype=torch.uint8, device=_DEV)
    b.awe_kv_attention(h, cache, s["rows"], types[s["type"]], s["T"], Hq, (Hq + 2 * H) * D, s["start"], s["ctx"], s["B"],
                       s["table"], s["width"], s["width"], s["scale"], True, s["window"], s["out"], Hq * D, s["lse"],
                       s["workspace"], s["workspace_bytes"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_w4(s):
    b, h, types = _library()
    if "matrix" not in s:
        s["matrix"] = b.w4_matrix(s["codes"], s["scale"], types[s["type"]], s["zero"], s["N"], s["K"], s["ld"], s["group"])
    b.awe_linear_w4(h, s["matrix"], s["x"], types[s["type"]], s["M"], s["K"], s["y"], types[s["out"]], s["N"])
    return s["y"]


def run(state):
    if own:
        return {"plan": _own_plan, "write": _own_write, "attn": _own_attn, "w4": _own_w4}[state["op"]](state)
    return {"plan": _plain_plan, "write": _plain_write, "attn": _plain_attn, "w4": _plain_w4}[state["op"]](state)


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    op = case["op"]
    if op == "plan":
        return None  # whole numbers only
    s = prepare(case, seed)
    if op == "w4":
        y = torch.zeros((s["M"], s["N"]), dtype=torch.float64, device=_DEV)
        low = (s["codes"].to(torch.int16) << 12).view(torch.int16) >> 12
        high = (s["codes"].to(torch.int16) << 8).view(torch.int16) >> 12
        q = torch.empty((s["N"], s["ld"]), dtype=torch.float64, device=_DEV)
        q[:, 0::2], q[:, 1::2] = low.double(), high.double()
        for j in range(s["scale"].shape[1]):
            a, b = j * s["group"], min(s["K"], (j + 1) * s["group"])
            part = q[:, a:b] - (s["zero"][:, j:j + 1].double() if s["zero"] is not None else 0.0)
            y += (s["x"][:, a:b].double() @ part.t()) * s["scale"][:, j].double()
        return y
    H, D, page = s["H"], s["D"], s["page"]
    if op == "write":
        slots, got = s["slots"], {"k": None, "v": None}
        for name, at in (("ks", 4), ("vs", 5)):
            x = s["rows"][:, at * H * D:(at + 1) * H * D].double().view(-1, H, D).abs().amax(2)
            scale = s[name].double()
            fresh = slots[slots % page == 0] // page
            scale[fresh] = 0.0  # nothing was there before
            scale.scatter_reduce_(0, (slots // page)[:, None].expand(-1, H), x / 127.0, "amax")
            got[name] = scale
        return got
    Hq, G = s["Hq"], s["Hq"] // H
    out = torch.zeros((s["T"], Hq, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device=_DEV)
    starts, lengths = s["start"].tolist(), s["ctx"].tolist()
    for i, length in enumerate(lengths):
        a, b = starts[i], starts[i + 1]
        pages = s["table"][i, :-(-length // page)].long()
        tok = torch.arange(length, device=_DEV)
        pos = torch.arange(length - (b - a), length, device=_DEV)[:, None]
        seen = tok <= pos
        if s["window"]:
            seen &= tok > pos - s["window"]
        for j in range(H):
            k = (s["k"][pages, j].double() * s["ks"][pages, j].double()[:, None, None]).view(-1, D)[:length]
            v = (s["v"][pages, j].double() * s["vs"][pages, j].double()[:, None, None]).view(-1, D)[:length]
            for head in range(j * G, (j + 1) * G):
                x = s["rows"][a:b, head * D:(head + 1) * D].double() @ k.t() * s["scale"]
                x = x.masked_fill(~seen, -math.inf)
                lse[a:b, head] = torch.logsumexp(x, 1)
                out[a:b, head] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
