"""Cases and plain forms of further serving operators: appending rotated keys and values to a paged cache of 4 bits (and
reading them back), the attention that reads that cache, low-rank adapters of many requests beside a shared projection, and
log probabilities of given tokens with entropy and top alternatives.

Each case is one pass through one operator.  `run` computes it with elementary torch operations in 32 bits (`own` false) or
with the library's entry points (`own` true); `exact` computes it from its definition in 64 bits.  Request lengths follow
from the case alone (`_lengths`), the seed orders them and fills the data.
"""
import math

import torch

own = False

_FLOAT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
_DEV = "cuda"


def listed():
    return [
        # one new token for each of 64 conversations of up to 8,191 tokens: every step of a decode loop
        {"name": "append_decode", "op": "append", "B": 64, "new": 1, "cached": 8191, "q_heads": 32, "heads": 8, "dim": 128,
         "page": 16, "rotary": 128, "interleaved": False, "type": "bf16", "ragged": True},
        # prompts of 1 to 4,095 tokens that start wherever the page before them ended; half of each head is rotated, in neighbours
        {"name": "append_prompts", "op": "append", "B": 9, "new": 4095, "cached": 333, "q_heads": 32, "heads": 8, "dim": 128,
         "page": 64, "rotary": 64, "interleaved": True, "type": "f16", "ragged": True},
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
        # one token of one user, an adapter of high rank on a large projection: latency
        {"name": "adapters_token", "op": "adapters", "B": 1, "new": 1, "adapters": 4, "rank": 64, "N": 8192, "K": 8192,
         "type": "bf16", "out": "bf16", "ragged": False},
        # a decode step of a full batch, most requests with an adapter of their own
        {"name": "adapters_batch", "op": "adapters", "B": 64, "new": 1, "adapters": 48, "rank": 16, "N": 4096, "K": 4096,
         "type": "bf16", "out": "bf16", "ragged": False},
        # prompts of 1 to 1,100 tokens, sizes that no tile divides
        {"name": "adapters_prompts", "op": "adapters", "B": 8, "new": 1100, "adapters": 6, "rank": 24, "N": 5003, "K": 4104,
         "type": "f16", "out": "f32", "ragged": True},
        # the answer to one user: the sampled token and five alternatives
        {"name": "logprobs_token", "op": "logprobs", "T": 1, "V": 32000, "top": 5, "temperature": 0.7, "pad": 0, "type": "f32"},
        # a decode step of a full batch over a large vocabulary
        {"name": "logprobs_batch", "op": "logprobs", "T": 128, "V": 131072, "top": 20, "temperature": 1.0, "pad": 0, "type": "bf16"},
        # scoring a prompt: every token's probability, an odd vocabulary in padded rows
        {"name": "logprobs_prompt", "op": "logprobs", "T": 2048, "V": 50257, "top": 1, "temperature": 1.0, "pad": 47, "type": "f16"},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "adapters", "adapters", "logprobs", "logprobs"])
    if op == "append":
        heads, dim, ratio = rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 256]), rng.choice([1, 4, 5, 8])
        new = _log(rng, 1, 4095)
        most = max(1, min(64, 24_000_000 // (new * heads * (ratio + 2) * dim)))
        return {"op": op, "B": _log(rng, 1, most), "new": new, "cached": _log(rng, 1, 8191) if rng.random() < 0.7 else 0,
                "q_heads": heads * ratio, "heads": heads, "dim": dim, "page": rng.choice([16, 32, 64, 128]),
                "rotary": rng.choice([dim, dim, dim // 2, 48]), "interleaved": rng.random() < 0.4, "type": rng.choice(["f16", "bf16"]),
                "ragged": rng.random() < 0.8}
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
    if op == "adapters":
        single = rng.random() < 0.5
        N, K, rank = _log(rng, 250, 8192), 8 * _log(rng, 32, 1024), 8 * _log(rng, 1, 16)
        new = 1 if single else _log(rng, 2, 1100)
        most = max(1, min(64, 40_000_000 // (new * (N + K)), 8_000_000 // (rank * (N + K))))
        return {"op": op, "B": _log(rng, 1, most), "new": new, "adapters": _log(rng, 1, 48), "rank": rank, "N": N, "K": K,
                "type": rng.choice(["f16", "bf16"]), "out": rng.choice(["same", "same", "f32"]), "ragged": rng.random() < 0.7}
    V = _log(rng, 1000, 150_000)
    return {"op": op, "T": _log(rng, 1, min(2048, 16_000_000 // V)), "V": V, "top": rng.choice([0, 1, _log(rng, 2, 32)]),
            "temperature": rng.choice([1.0, 0.6, 1.5]), "pad": rng.choice([0, 0, 1, 16]), "type": rng.choice(["f16", "bf16", "f32"])}


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
    if case["op"] == "adapters" or case["cached"] == 0:
        return [0] * B, new
    return _lengths(B, case["cached"], case["ragged"])[::-1], new


def work(case):
    op = case["op"]
    if op == "logprobs":
        T, V, k = case["T"], case["V"], case["top"]
        # the logits and the tokens in; three numbers a row and the alternatives out
        return {"bytes": T * V * (4 if case["type"] == "f32" else 2) + T * (4 + 12 + 8 * k), "flops": 6 * T * V}
    cached, new = _requests(case)
    T = sum(new)
    if op == "adapters":
        N, K, r, out = case["N"], case["K"], case["rank"], 4 if case["out"] == "f32" else 2
        used = min(case["adapters"], case["B"])  # adapters that some request reads
        # rows and the shared projection's result in, the sum out, each adapter in use once
        return {"bytes": T * (2 * K + 2 * out * N) + used * r * 2 * (N + K) + 8 * case["B"], "flops": 2 * T * r * (N + K)}
    page, H, D, Hq = case["page"], case["heads"], case["dim"], case["q_heads"]
    if op == "append":
        # rows, slots, positions and their angles in; rotated queries, codes and parameters out; then those in again, FP16 values out
        return {"bytes": T * (2 * (Hq + 2 * H) * D + 12 + 4 * case["rotary"] + 2 * Hq * D + 2 * 2 * H * (D // 2 + 2) + 2 * 2 * H * D),
                "flops": T * (Hq * 3 * D + H * 3 * D + 2 * H * 6 * D)}
    window = case["window"]
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
    return {"bytes": tokens * 2 * H * (D // 2 + 2) + pages * 4 + T * Hq * (4 * D + 4) + 8 * case["B"], "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + 13)


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.float32, device=_DEV).normal_(generator=g)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEV)


def _pool(g, pages, heads, page, dim):
    """Keys or values as a cache of 4 bits holds them: two signed codes a byte, the even dimension in the low half, and for each
    token and head 16 bits: FP16 of 16 times the scale, the lowest four bits replaced by the zero point."""
    zero = torch.randint(-3, 3, (pages, heads, page), generator=g, device=_DEV, dtype=torch.int16)
    scale = _normal(g, pages, heads, page).mul_(0.25).exp_().mul_(0.3)
    code = torch.empty((pages, heads, page, dim), dtype=torch.float16, device=_DEV).normal_(0.0, 2.7, generator=g)
    code = code.add_(zero[..., None]).round_().clamp_(-8, 7).to(torch.int8)
    codes = ((code[..., 0::2] & 15) | (code[..., 1::2] << 4)).view(torch.uint8)
    return codes, ((scale * 16.0).to(torch.float16).view(torch.int16) & -16) | (zero & 15)


def _angles(count, dim):
    """cos and sin of position times 10000^(-2 i / dim), from 64 bits."""
    step = torch.exp(torch.arange(0, dim, 2, dtype=torch.float64, device=_DEV) * (-math.log(10000.0) / dim))
    angle = torch.arange(count, dtype=torch.float64, device=_DEV)[:, None] * step
    return torch.cat([torch.cos(angle), torch.sin(angle)], 1).to(torch.float32)


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    if op == "logprobs":
        T, V, t = case["T"], case["V"], _FLOAT[case["type"]]
        ld = V + case["pad"]
        x = _normal(g, T, ld).mul_(2.0)
        x += _normal(g, T, 1)
        # a few likely tokens stand out, and some are forbidden
        likely = torch.randint(0, V, (T, 12), generator=g, device=_DEV)
        x.scatter_add_(1, likely, _normal(g, T, 12).abs_().mul_(4.0))
        x.scatter_(1, torch.randint(0, V, (T, 5), generator=g, device=_DEV), -math.inf)
        at = torch.randint(0, 12, (T, 1), generator=g, device=_DEV)
        k = case["top"]
        return {"op": op, "T": T, "V": V, "ld": ld, "top": k, "type": case["type"], "scale": 1.0 / case["temperature"],
                "logits": x.to(t), "tokens": likely.gather(1, at)[:, 0].to(torch.int32),
                "logprob": torch.empty(T, device=_DEV), "entropy": torch.empty(T, device=_DEV), "lse": torch.empty(T, device=_DEV),
                "top_logprob": torch.empty((T, k), device=_DEV), "top_id": torch.empty((T, k), dtype=torch.int32, device=_DEV)}
    cached, new = _requests(case)
    B, t = case["B"], _FLOAT[case["type"]]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed))).tolist()
    cached, new = [cached[i] for i in order], [new[i] for i in order]
    T = sum(new)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    if op == "adapters":
        N, K, r, L = case["N"], case["K"], case["rank"], case["adapters"]
        out = case["type"] if case["out"] == "same" else case["out"]
        which = torch.randperm(max(L, B), generator=g, device=_DEV)[:B] % L
        if B > 4:
            which[0] = -1  # one request without an adapter
        return {"op": op, "B": B, "T": T, "N": N, "K": K, "rank": r, "L": L, "most_new": max(new), "type": case["type"], "out": out,
                "start": _ints(starts), "which": which.to(torch.int32), "x": _normal(g, T, K).to(t),
                "a": _normal(g, L, r, K).mul_(K ** -0.5).to(t), "b": _normal(g, L, N, r).mul_(r ** -0.5).to(t),
                "scale": torch.rand(L, generator=g, device=_DEV) + 0.5, "base": _normal(g, T, N).to(_FLOAT[out]),
                "y": torch.empty((T, N), dtype=_FLOAT[out], device=_DEV)}
    page, H, D, Hq = case["page"], case["heads"], case["dim"], case["q_heads"]
    # block tables over a shuffled pool, with room for the call's own tokens
    want = [-(-(c + n) // page) for c, n in zip(cached, new)]
    width, pool = max(want) + 1, sum(want) + 8
    free = torch.randperm(pool, generator=g, device=_DEV).to(torch.int32)
    hold = torch.tensor(want, device=_DEV)
    first = torch.cumsum(hold, 0) - hold
    col = torch.arange(width, device=_DEV)
    table = torch.where(col < hold[:, None], free[(first[:, None] + col).clamp_(max=pool - 1)], -1).to(torch.int32)
    k, kp = _pool(g, pool, H, page, D)
    v, vp = _pool(g, pool, H, page, D)
    rows = _normal(g, T, (Hq + 2 * H) * D)
    s = {"op": op, "B": B, "T": T, "page": page, "H": H, "D": D, "Hq": Hq, "type": case["type"], "table": table, "width": width,
         "pool": pool, "k": k, "v": v, "kp": kp, "vp": vp, "start": _ints(starts)}
    if op == "append":
        request = torch.repeat_interleave(torch.arange(B, device=_DEV), torch.tensor(new, device=_DEV), output_size=T)
        pos = (torch.tensor(cached, device=_DEV) - s["start"][:-1])[request] + torch.arange(T, device=_DEV)
        rows *= _normal(g, 1, (Hq + 2 * H) * D).mul_(0.4).exp_()  # some channels are large, as in keys
        n_positions = max(c + n for c, n in zip(cached, new))
        s.update(rows=rows.to(t), slots=table[request, pos // page].long() * page + pos % page, positions=pos.to(torch.int32),
                 rotary=case["rotary"], interleaved=case["interleaved"], n_positions=n_positions,
                 angles=_angles(n_positions, case["rotary"]), q=torch.empty((T, Hq, D), dtype=t, device=_DEV),
                 k_out=torch.empty((T, H, D), dtype=torch.float16, device=_DEV),
                 v_out=torch.empty((T, H, D), dtype=torch.float16, device=_DEV))
        return s
    s.update(rows=rows.to(t), ctx=_ints([c + n for c, n in zip(cached, new)]), window=case["window"], scale=1.0 / math.sqrt(D),
             most_new=max(new), most_ctx=max(c + n for c, n in zip(cached, new)),
             out=torch.empty((T, Hq, D), dtype=t, device=_DEV), lse=torch.empty((T, Hq), dtype=torch.float32, device=_DEV))
    return s


# ------------------------------------------------------------------ plain forms
def _unpacked(codes, par):
    """The values that codes (..., dim / 2 bytes) and their parameters (...) stand for."""
    q = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float()
    zero = (par & 15).float()
    q, zero = torch.where(q > 7, q - 16, q), torch.where(zero > 7, zero - 16, zero)
    scale = (par & -16).view(torch.float16).float() * 0.0625
    return (q - zero[..., None]) * scale[..., None]


def _plain_rotated(x, cos, sin, interleaved):
    """x: T x heads x D in 32 bits; cos, sin: T x 1 x rotary / 2."""
    half = cos.shape[2]
    if interleaved:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_store(codes, par, x, slots, page):
    """Quantises x (T x H x D in 32 bits) into its slots."""
    lo, hi = x.amin(2).clamp(-30480.0, 0.0), x.amax(2).clamp(0.0, 30480.0)
    raw = (hi - lo).div(torch.full_like(lo, 15.0)).clamp(min=2.0 ** -18)
    scale = ((raw.view(torch.int32) + 0x1FFFF) & ~0x1FFFF).view(torch.float32)  # up to 7 significant bits
    below = (lo / scale).round()
    code = ((x / scale[..., None]).round() - below[..., None] - 8.0).clamp(-8.0, 7.0).to(torch.int8)
    of, at = slots // page, slots % page
    codes[of, :, at] = ((code[..., 0::2] & 15) | (code[..., 1::2] << 4)).view(torch.uint8)
    zero = (-below - 8.0).to(torch.int16)
    par[of, :, at] = ((scale * 16.0).to(torch.float16).view(torch.int16) & -16) | (zero & 15)


def _plain_append(s):
    Hq, H, D, T, page, slots = s["Hq"], s["H"], s["D"], s["T"], s["page"], s["slots"]
    half = s["rotary"] // 2
    angles = s["angles"][s["positions"].long()][:, None]
    cos, sin = angles[..., :half], angles[..., half:]
    rows = s["rows"].float().view(T, Hq + 2 * H, D)
    turned = _plain_rotated(rows[:, :Hq + H], cos, sin, s["interleaved"])
    _plain_store(s["k"], s["kp"], turned[:, Hq:], slots, page)
    _plain_store(s["v"], s["vp"], rows[:, Hq + H:], slots, page)
    of, at = slots // page, slots % page
    back = lambda codes, par: _unpacked(codes[of, :, at], par[of, :, at]).to(torch.float16)  # noqa: E731
    return {"q": turned[:, :Hq].to(_FLOAT[s["type"]]), "k": back(s["k"], s["kp"]), "v": back(s["v"], s["vp"])}


def _plain_attn(s):
    B, H, D, Hq, T, page = s["B"], s["H"], s["D"], s["Hq"], s["T"], s["page"]
    G, most = Hq // H, s["most_new"]
    pages = s["table"][:, :-(-s["most_ctx"] // page)].long().clamp(min=0)
    span = pages.shape[1] * page

    def gather(codes, par):
        return _unpacked(codes[pages], par[pages]).permute(0, 2, 1, 3, 4).reshape(B, H, span, D)

    start, ctx = s["start"].long(), s["ctx"].long()
    n = start[1:] - start[:-1]
    row = torch.arange(most, device=_DEV)
    q = s["rows"][:, :Hq * D].reshape(T, H, G, D)[(start[:-1, None] + row).clamp(max=T - 1)].float()
    q = q.permute(0, 2, 3, 1, 4).reshape(B, H, G * most, D)
    score = (q * s["scale"]) @ gather(s["k"], s["kp"]).transpose(2, 3)
    score = score.view(B, H, G, most, span)
    pos, tok = (ctx - n)[:, None] + row, torch.arange(span, device=_DEV)
    hidden = tok > pos[..., None]
    if s["window"]:
        hidden |= tok <= pos[..., None] - s["window"]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    m = score.amax(-1, keepdim=True).clamp(min=-3e38)
    p = score.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(B, H, G * most, span) @ gather(s["v"], s["vp"])).view(B, H, G, most, D) / total
    o = torch.where(total > 0, o, 0.0)
    lse = torch.where(total > 0, m + torch.log(total), -math.inf)[..., 0]
    request = torch.searchsorted(start[1:], torch.arange(T, device=_DEV), right=True)
    index = torch.arange(T, device=_DEV) - start[request]
    out = o.permute(0, 3, 1, 2, 4)[request, index].reshape(T, Hq, D)
    return {"out": out.to(_FLOAT[s["type"]]), "lse": lse.permute(0, 3, 1, 2)[request, index].reshape(T, Hq)}


def _plain_adapters(s):
    T, start, which = s["T"], s["start"].long(), s["which"].long()
    token = (start[:-1, None] + torch.arange(s["most_new"], device=_DEV)).clamp(max=T - 1)  # request by request, padded
    index = which.clamp(min=0)
    low = s["x"][token].float() @ s["a"][index].float().transpose(1, 2)
    part = (low @ s["b"][index].float().transpose(1, 2)) * s["scale"][index][:, None, None]
    part = torch.where((which >= 0)[:, None, None], part, 0.0)
    request = torch.searchsorted(start[1:], torch.arange(T, device=_DEV), right=True)
    return (s["base"].float() + part[request, torch.arange(T, device=_DEV) - start[request]]).to(_FLOAT[s["out"]])


def _plain_logprobs(s):
    V, k = s["V"], s["top"]
    logit = s["logits"][:, :V].float()
    m = logit.amax(1, keepdim=True)
    d = (logit - m) * s["scale"]
    e = torch.exp(d)
    total = e.sum(1, dtype=torch.float64)
    log_total = torch.log(total)
    mean = torch.where(e > 0, e * d, 0.0).sum(1, dtype=torch.float64) / total
    of = lambda x: ((x - m) * s["scale"] - log_total[:, None]).float()  # noqa: E731
    # larger first, then the lower index: both in one whole number
    bits = (logit + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    order = (order << 32) + (V - 1 - torch.arange(V, device=_DEV))
    ids = V - 1 - (torch.topk(order, k, 1).values & 0xFFFFFFFF) if k else order[:, :0]
    return {"logprob": of(logit.gather(1, s["tokens"].long()[:, None]))[:, 0], "entropy": (log_total - mean).float(),
            "lse": (m[:, 0].double() * s["scale"] + log_total).float(), "top_logprob": of(logit.gather(1, ids)),
            "top_id": ids.to(torch.int32)}


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
        s["cache"] = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], s["H"], s["page"], s["D"])
    return s["cache"]


def _own_append(s):
    b, h, types = _library()
    cache, H, D, Hq, T, rows = _cache(b, s), s["H"], s["D"], s["Hq"], s["T"], s["rows"]
    if "turn" not in s:
        s["turn"] = b.rotary(s["angles"], s["n_positions"], s["rotary"], s["interleaved"])
        s["keys"], s["values"] = rows[:, Hq * D:], rows[:, (Hq + H) * D:]
    ld = (Hq + 2 * H) * D
    b.awe_kv4_append(h, cache, s["turn"], types[s["type"]], T, Hq, rows, ld, s["keys"], ld, s["values"], ld, s["positions"], s["slots"],
                     s["q"], Hq * D)
    b.awe_kv4_read(h, cache, T, s["slots"], b.F16, s["k_out"], H * D, s["v_out"], H * D)
    return {"q": s["q"], "k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    b, h, types = _library()
    cache, H, D, Hq = _cache(b, s), s["H"], s["D"], s["Hq"]
    if "workspace" not in s:
        s["workspace_bytes"] = b.awe_kv4_attention_workspace_bytes(h, cache, s["T"], Hq, s["B"])
        s["workspace"] = torch.empty(max(1, s["workspace_bytes"]), dtype=torch.uint8, device=_DEV)
    b.awe_kv4_attention(h, cache, s["rows"], types[s["type"]], s["T"], Hq, (Hq + 2 * H) * D, s["start"], s["ctx"], s["B"],
                        s["table"], s["width"], s["width"], s["scale"], True, s["window"], s["out"], Hq * D, s["lse"],
                        s["workspace"], s["workspace_bytes"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_adapters(s):
    b, h, types = _library()
    if "adapters" not in s:
        s["adapters"] = b.adapters(s["a"], s["b"], s["scale"], types[s["type"]], s["L"], s["rank"], s["N"], s["K"])
    b.awe_linear_adapters(h, s["adapters"], s["x"], s["T"], s["K"], s["start"], s["which"], s["B"], s["base"], s["N"], s["y"],
                          types[s["out"]], s["N"])
    return s["y"]


def _own_logprobs(s):
    b, h, types = _library()
    b.awe_token_logprobs(h, s["logits"], types[s["type"]], s["T"], s["V"], s["ld"], s["scale"], s["tokens"], s["logprob"], s["entropy"],
                         s["lse"], s["top"], s["top_logprob"], s["top_id"])
    return {"logprob": s["logprob"], "entropy": s["entropy"], "lse": s["lse"], "top_logprob": s["top_logprob"], "top_id": s["top_id"]}


def run(state):
    if own:
        return {"append": _own_append, "attn": _own_attn, "adapters": _own_adapters, "logprobs": _own_logprobs}[state["op"]](state)
    return {"append": _plain_append, "attn": _plain_attn, "adapters": _plain_adapters, "logprobs": _plain_logprobs}[state["op"]](state)


# ------------------------------------------------------------------ 64 bits
def _exact_quantised(x):
    """Per row of 64-bit x: the multiple of its scale that stands for each value."""
    lo = torch.clamp(x.amin(-1, keepdim=True), -30480.0, 0.0)
    raw = torch.clamp((torch.clamp(x.amax(-1, keepdim=True), 0.0, 30480.0) - lo) / 15.0, min=2.0 ** -18)
    unit = torch.exp2(torch.floor(torch.log2(raw)) - 6.0)
    scale = torch.ceil(raw / unit) * unit
    lowest = torch.round(lo / scale)
    return torch.minimum(torch.round(x / scale), lowest + 15.0).maximum(lowest) * scale


def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op == "logprobs":
        T, V, k = s["T"], s["V"], s["top"]
        got = {"logprob": [], "entropy": [], "lse": [], "top_logprob": []}
        for a in range(0, T, 256):
            x = s["logits"][a:a + 256, :V].double() * s["scale"]
            logp = torch.log_softmax(x, 1)
            got["logprob"].append(logp.gather(1, s["tokens"][a:a + 256].long()[:, None])[:, 0])
            got["entropy"].append(-torch.where(logp > -math.inf, logp.exp() * logp, 0.0).sum(1))
            got["lse"].append(torch.logsumexp(x, 1))
            got["top_logprob"].append(logp.topk(k, 1).values)
        return {**{name: torch.cat(parts) for name, parts in got.items()}, "top_id": None}
    if op == "adapters":
        y = s["base"].double()
        starts, which = s["start"].tolist(), s["which"].tolist()
        for i, j in enumerate(which):
            if j >= 0:
                a, b = starts[i], starts[i + 1]
                y[a:b] += s["scale"][j].double() * ((s["x"][a:b].double() @ s["a"][j].double().t()) @ s["b"][j].double().t())
        return y
    H, D, page, Hq = s["H"], s["D"], s["page"], s["Hq"]
    if op == "append":
        x = s["rows"].double().view(s["T"], Hq + 2 * H, D)
        half = s["rotary"] // 2
        table = s["angles"][s["positions"].long()].double()
        turn = torch.complex(table[:, :half], table[:, half:])[:, None]
        at = torch.arange(2 * half, device=_DEV).view(half, 2) if s["interleaved"] else torch.arange(2 * half, device=_DEV).view(2, half).t()
        z = torch.complex(x[:, :Hq + H, at[:, 0]], x[:, :Hq + H, at[:, 1]]) * turn
        x[:, :Hq + H, at[:, 0]], x[:, :Hq + H, at[:, 1]] = z.real, z.imag
        return {"q": x[:, :Hq], "k": _exact_quantised(x[:, Hq:Hq + H]), "v": _exact_quantised(x[:, Hq + H:])}
    G = Hq // H
    out = torch.zeros((s["T"], Hq, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((s["T"], Hq), -math.inf, dtype=torch.float64, device=_DEV)
    starts, lengths = s["start"].tolist(), s["ctx"].tolist()

    def values(codes, par, pages, head, length):
        c, p = codes[pages, head].flatten(0, 1)[:length].to(torch.int32), par[pages, head].flatten()[:length].to(torch.int32)
        x = torch.empty((length, D), dtype=torch.float64, device=_DEV)
        zero = ((p & 15) ^ 8) - 8
        x[:, 0::2], x[:, 1::2] = (((c & 15) ^ 8) - 8 - zero[:, None]).double(), (((c >> 4) ^ 8) - 8 - zero[:, None]).double()
        return x * ((p & 0xFFF0).to(torch.int16).view(torch.float16).double() / 16.0)[:, None]

    for i, length in enumerate(lengths):
        a, b = starts[i], starts[i + 1]
        pages = s["table"][i, :-(-length // page)].long()
        tok = torch.arange(length, device=_DEV)
        pos = torch.arange(length - (b - a), length, device=_DEV)[:, None]
        seen = tok <= pos
        if s["window"]:
            seen &= tok > pos - s["window"]
        for j in range(H):
            k, v = values(s["k"], s["kp"], pages, j, length), values(s["v"], s["vp"], pages, j, length)
            for head in range(j * G, (j + 1) * G):
                x = s["rows"][a:b, head * D:(head + 1) * D].double() @ k.t() * s["scale"]
                x = x.masked_fill(~seen, -math.inf)
                lse[a:b, head] = torch.logsumexp(x, 1)
                out[a:b, head] = torch.softmax(x, 1) @ v
    return {"out": out, "lse": lse}
