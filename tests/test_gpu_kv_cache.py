"""The paged 8-bit cache: plan, write and attention against plain implementations on the host.

Tolerances.  Whole numbers, and the stored cache (whose rounding is specified to the bit), are equal.  For the
attention, with u the unit roundoff of the output type and A = sum_j p_j |v_j| (64 bits): the weights are rounded to FP16
(relative 2^-11, or 2^-25 absolute where they are below its normal range) both above and below the fraction, and the
scores carry the error of FP32 sums of D / 16 matrix steps, each at most 2^-22 of the sum of magnitudes S, so
  |out - ref| <= u |ref| + (2^-11 + e) (A + |ref|) + n 2^-24 max|v|,   |lse - ref| <= e + 2^-21 (1 + |ref|),
  e = 2 (D / 16 + 3) 2^-22 S.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_24519_b200 import binding as b
from tests.gpu_util import handle

pytestmark = pytest.mark.gpu

TYPES = {"f16": (b.F16, torch.float16, 2.0 ** -11), "bf16": (b.BF16, torch.bfloat16, 2.0 ** -8)}


def cuda(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


# ------------------------------------------------------------------ plan
def plain_plan(cached, new, page, free, table, max_tokens):
    table, at = table.copy(), 0
    slots, positions, start, ctx, missing = [], [], [0], [], 0
    for i, (c, n) in enumerate(zip(cached, new)):
        c, n = max(int(c), 0), max(int(n), 0)
        have, want = -(-c // page), -(-(c + n) // page)
        for j in range(have, want):
            if j < table.shape[1]:
                table[i, j] = free[at] if at < len(free) else -1
                missing += at >= len(free)
                at += 1
            else:
                missing += 1
        for pos in range(c, c + n):
            p = table[i, pos // page] if pos // page < table.shape[1] else -1
            slots.append(int(p) * page + pos % page if p >= 0 else -1)
            positions.append(pos)
        start.append(start[-1] + n)
        ctx.append(c + n)
    counts = [min(at, len(free)), start[-1], missing, max(ctx, default=0)]
    pad = max(0, max_tokens - len(slots))
    return (table, np.array(slots + [-1] * pad, np.int64)[:max_tokens], np.array(positions + [-1] * pad, np.int32)[:max_tokens],
            np.array(start, np.int32), np.array(ctx, np.int32), np.array(counts, np.int32))


def run_plan(cached, new, page, free, table, max_tokens, ld_extra=0, positions=True):
    B, width = table.shape
    wide = np.full((B, width + ld_extra), 99, np.int32)
    wide[:, :width] = table
    d = dict(cached=cuda(np.array(cached, np.int32)), new=cuda(np.array(new, np.int32)), free=cuda(np.array(free, np.int32)),
             table=cuda(wide), slots=torch.full((max_tokens + 3,), 77, dtype=torch.int64, device="cuda"),
             positions=torch.full((max_tokens + 3,), 77, dtype=torch.int32, device="cuda") if positions else None,
             start=torch.full((B + 1,), 77, dtype=torch.int32, device="cuda"),
             ctx=torch.full((max(B, 1),), 77, dtype=torch.int32, device="cuda"),
             counts=torch.full((4,), 77, dtype=torch.int32, device="cuda"))
    for _ in range(2):  # the same again with the same arguments
        b.awe_kv_plan(handle(), d["cached"], d["new"], B, page, d["free"], len(free), d["table"], width, width + ld_extra,
                      d["slots"], d["positions"], max_tokens, d["start"], d["ctx"], d["counts"])
    torch.cuda.synchronize()
    got = {k: v.cpu().numpy() for k, v in d.items() if v is not None}
    assert (got["table"][:, width:] == 99).all() and (got["slots"][max_tokens:] == 77).all()
    return got


@pytest.mark.parametrize("B,page,most_cached,most_new,short", [
    (1, 16, 0, 1, 0), (1, 16, 16, 1, 0), (1, 256, 255, 2, 0), (7, 16, 40, 40, 0), (64, 16, 4096, 1, 0),
    (300, 32, 0, 700, 0), (33, 64, 100, 300, 5), (33, 16, 100, 300, 100000), (1000, 128, 3000, 1, 7), (5000, 16, 50, 3, 0)])
def test_plan(B, page, most_cached, most_new, short):
    rng = np.random.default_rng(B * 1000 + page)
    cached = rng.integers(-2 if B > 1 else 0, most_cached + 1, B)
    new = rng.integers(-1 if B > 5 else 1, most_new + 1, B)
    if B > 5:
        new[0], cached[1], new[1] = 0, 0, 0
    have = np.maximum(-(-np.maximum(cached, 0) // page), 0)
    want = -(-(np.maximum(cached, 0) + np.maximum(new, 0)) // page)
    width = max(int(want.max()) - (1 if short else 0), int(have.max()), 1)
    table = rng.integers(0, 10 ** 6, (B, width)).astype(np.int32)
    if B > 5:
        table[2, :] = -1  # pages that are gone: their tokens have no slot
    free = rng.permutation(max(0, int((want - have).sum()) - short) + (0 if short else 3)).astype(np.int32)
    total = int(np.maximum(new, 0).sum())
    for max_tokens in (total + 9, max(total - 5, 0)):
        got = run_plan(cached, new, page, free, table, max_tokens, ld_extra=3)
        want_out = plain_plan(cached, new, page, free, table, max_tokens)
        for name, w in zip(("table", "slots", "positions", "start", "ctx", "counts"), want_out):
            assert np.array_equal(got[name][..., :w.shape[-1]] if name in ("table", "slots", "positions") else got[name], w), name


def test_plan_of_no_requests_and_without_positions():
    got = run_plan([], [], 16, [1, 2], np.zeros((0, 4), np.int32), 5)
    assert got["start"].tolist() == [0] and got["counts"].tolist() == [0, 0, 0, 0] and (got["slots"][:5] == -1).all()
    got = run_plan([3], [2], 16, [], np.array([[7]], np.int32), 2, positions=False)
    assert got["slots"][:2].tolist() == [7 * 16 + 3, 7 * 16 + 4]


# ------------------------------------------------------------------ write
def plain_write(cache, scale, x, slots, page):
    """Token run by token run, in FP32 with the specified roundings."""
    f = np.float32
    t = 0
    while t < len(slots):
        if slots[t] < 0 or slots[t] // page >= cache.shape[0]:
            t += 1
            continue
        p, e = slots[t] // page, t
        while e < len(slots) and slots[e] // page == p and slots[e] >= 0:
            e += 1
        place = int(slots[t] % page)
        for h in range(cache.shape[1]):
            rows = x[t:e, h].astype(f)
            finite = np.isfinite(rows)
            a = f(np.abs(np.where(finite, rows, f(0))).max())
            wanted = f(0) if a < f(2.0 ** -100) else a * (f(1) / f(127))
            before = scale[p, h] if place else f(0)
            after = max(before, wanted)
            if after > before and place:
                cache[p, h, :place] = np.rint(cache[p, h, :place].astype(f) * (before / after)).astype(np.int8)
            inverse = f(1) / after if after > 0 else f(0)
            q = np.rint(np.where(finite, rows, f(0)) * inverse)
            q = np.where(np.isnan(rows), f(0), np.where(finite, q, np.sign(rows) * f(127)))
            for i, s in enumerate(slots[t:e]):
                cache[p, h, s % page] = np.clip(q[i], -127, 127).astype(np.int8)
            scale[p, h] = after
        t = e


@pytest.mark.parametrize("heads,dim,page,kind", [(1, 64, 16, "f16"), (3, 128, 16, "bf16"), (8, 128, 64, "bf16"), (2, 256, 256, "f16"),
                                                 (5, 64, 128, "bf16"), (1, 256, 32, "bf16")])
@pytest.mark.parametrize("offset", [0, 1])  # 1: rows that no 16-byte load can take
def test_write(heads, dim, page, kind, offset):
    rng = np.random.default_rng(heads * dim + page)
    enum, dtype, _ = TYPES[kind]
    cached = [0, 0, 5, page - 1, page, 3 * page + 7, 0, 2 * page - 3, 1]
    new = [1, page + 1, 3, 2, 1, 2 * page, 0, page // 2, 1]
    need = [-(-(c + n) // page) for c, n in zip(cached, new)]
    n_pages = sum(need) + 4
    pages, at, slots = rng.permutation(n_pages), 0, []
    for c, n, k in zip(cached, new, need):
        slots += [int(pages[at + pos // page]) * page + pos % page for pos in range(c, c + n)]
        at += k
    slots += [-1, n_pages * page, -5]
    T = len(slots)
    ld = 2 * heads * dim + (8 if not offset else 3)
    x = torch.from_numpy(rng.standard_normal((T, ld)).astype(np.float32) * 3).to(dtype)
    k, v = x[:, offset:offset + heads * dim], x[:, offset + heads * dim:offset + 2 * heads * dim]
    k[1] = 0  # a first token of nothing but zeros
    k[3, :5] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1e-30, -1e-30]).to(dtype)
    v[4] *= 2.0 ** -14  # small beside what follows
    v[6] *= 50.0        # grows a page that is partly filled
    caches = [rng.integers(-127, 128, (n_pages, heads, page, dim)).astype(np.int8) for _ in range(2)]
    scales = [np.abs(rng.standard_normal((n_pages, heads))).astype(np.float32) * 0.02 for _ in range(2)]
    scales[0][pages[2], :] = 0.0
    dev = [cuda(c) for c in caches] + [cuda(s) for s in scales]
    c = b.kv_cache(*dev, n_pages, heads, page, dim)
    dx, ds = x.cuda(), cuda(np.array(slots, np.int64))
    for _ in range(2):  # writing the same tokens again changes nothing
        b.awe_kv_write(handle(), c, dx[:, offset:], dx[:, offset + heads * dim:], enum, T, ld, ld, ds)
        torch.cuda.synchronize()
        if _ == 0:
            for cache, scale, rows in zip(caches, scales, (k, v)):
                plain_write(cache, scale, rows.float().numpy().reshape(T, heads, dim), slots, page)
        for want, got in zip(caches + scales, dev):
            assert np.array_equal(want, got.cpu().numpy())


def test_write_with_places_left_out():
    """Tokens of a page that leave places out: those keep what they had."""
    rng = np.random.default_rng(1)
    heads, dim, page, n_pages = 2, 64, 32, 3
    slots = [2 * page, 2 * page + 1, 2 * page + 5, 2 * page + 31, 4, 6, 7]
    x = torch.from_numpy(rng.standard_normal((len(slots), heads * dim)).astype(np.float32)).to(torch.float16)
    cache, scale = rng.integers(-127, 128, (n_pages, heads, page, dim)).astype(np.int8), np.full((n_pages, heads), 0.01, np.float32)
    dev = [cuda(cache), cuda(cache), cuda(scale), cuda(scale)]
    b.awe_kv_write(handle(), b.kv_cache(*dev, n_pages, heads, page, dim), x.cuda(), x.cuda(), b.F16, len(slots), heads * dim, heads * dim,
                   cuda(np.array(slots, np.int64)))
    plain_write(cache, scale, x.float().numpy().reshape(-1, heads, dim), slots, page)
    for want, got in zip((cache, cache, scale, scale), dev):
        assert np.array_equal(want, got.cpu().numpy())


def test_write_many_tokens_is_within_half_a_step():
    rng = torch.Generator(device="cuda").manual_seed(3)
    T, heads, dim, page = 20000, 4, 128, 32
    n_pages = -(-T // page)
    x = torch.empty((T, 2, heads, dim), device="cuda").normal_(generator=rng).to(torch.bfloat16)
    k, v = (torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((n_pages, heads), device="cuda") for _ in range(2))
    slots = torch.arange(T, device="cuda")
    b.awe_kv_write(handle(), b.kv_cache(k, v, ks, vs, n_pages, heads, page, dim), x, x[:, 1], b.BF16, T, 2 * heads * dim,
                   2 * heads * dim, slots)
    for i, (q, s) in enumerate(((k, ks), (v, vs))):
        back = (q.double() * s.double()[..., None, None]).permute(0, 2, 1, 3).reshape(-1, heads, dim)[:T]
        step = s.double()[torch.arange(T, device="cuda") // page][..., None]
        assert bool(((back - x[:, i].double()).abs() <= step * (0.5 + 127 * 2.0 ** -22)).all())


# ------------------------------------------------------------------ attention
def make_cache(rng, n_pages, heads, page, dim):
    k, v = (rng.integers(-127, 128, (n_pages, heads, page, dim)).astype(np.int8) for _ in range(2))
    ks, vs = ((np.exp(rng.standard_normal((n_pages, heads)) * 0.5) * 0.02).astype(np.float32) for _ in range(2))
    return k, v, ks, vs


def plain_attention(cache, q, start, ctx, table, scale, causal, window):
    """In 64 bits; returns out, lse and the bound on each of the module's docstring (without u)."""
    k, v, ks, vs = cache
    n_pages, heads, page, dim = k.shape
    T, Hq, _ = q.shape
    group = Hq // heads
    out, lse = np.zeros((T, Hq, dim)), np.full((T, Hq), -np.inf)
    out_tol, lse_tol = np.full((T, Hq, dim), 1e-30), np.zeros((T, Hq))
    for i in range(len(ctx)):
        for t in range(start[i], start[i + 1]):
            place = ctx[i] - (start[i + 1] - start[i]) + t - start[i]
            hi = min(place + 1, ctx[i]) if causal else ctx[i]
            lo = max(0, place + 1 - window) if window else 0
            tok = np.arange(lo, max(hi, lo))
            tok = tok[tok // page < table.shape[1]]
            pages = table[i, tok // page]
            fine = (pages >= 0) & (pages < n_pages)
            tok, pages = tok[fine], pages[fine]
            if not len(tok):
                continue
            for h in range(heads):
                K = k[pages, h, tok % page].astype(float) * ks[pages, h][:, None]
                V = v[pages, h, tok % page].astype(float) * vs[pages, h][:, None]
                for j in range(h * group, (h + 1) * group):
                    s = K @ q[t, j] * scale
                    m = s.max()
                    p = np.exp(s - m)
                    out[t, j] = p @ V / p.sum()
                    lse[t, j] = m + np.log(p.sum())
                    e = 2 * (dim / 16 + 3) * 2.0 ** -22 * np.abs(K * q[t, j]).sum(1).max() * abs(scale)
                    A = p @ np.abs(V) / p.sum()
                    out_tol[t, j] = (2.0 ** -11 + e) * (A + np.abs(out[t, j])) + len(tok) * 2.0 ** -24 * np.abs(V).max()
                    lse_tol[t, j] = e + 2.0 ** -21 * (1 + abs(lse[t, j]))
    return out, lse, out_tol, lse_tol


def run_attention(cache, q, kind, start, ctx, table, scale, causal=True, window=0, ld_extra=0, with_lse=True):
    n_pages, heads, page, dim = cache[0].shape
    T, Hq, _ = q.shape
    enum, dtype, _ = TYPES[kind]
    ld = Hq * dim + ld_extra
    dq = torch.zeros((T, ld), dtype=dtype, device="cuda")
    dq[:, :Hq * dim] = q.reshape(T, -1).cuda()
    out = torch.full((T, ld), 77.0, dtype=dtype, device="cuda")
    lse = torch.full((T, Hq), 77.0, device="cuda") if with_lse else None
    dev = [cuda(x) for x in cache]
    c = b.kv_cache(*dev, n_pages, heads, page, dim)
    n = b.awe_kv_attention_workspace_bytes(handle(), c, T, Hq, len(ctx))
    work = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # nothing in it is taken for granted
    b.awe_kv_attention(handle(), c, dq, enum, T, Hq, ld, cuda(np.array(start, np.int32)), cuda(np.array(ctx, np.int32)), len(ctx),
                       cuda(table.astype(np.int32)), table.shape[1], table.shape[1], scale, causal, window, out, ld, lse, work)
    torch.cuda.synchronize()
    assert b.awe_last_device_status(handle()) == (0, 0)
    if ld_extra:
        assert bool((out[:, Hq * dim:] == 77).all())
    return out[:, :Hq * dim].double().cpu().numpy().reshape(T, Hq, dim), lse.double().cpu().numpy() if with_lse else None


def check_attention(rng, heads, group, dim, page, kind, new, ctx, causal=True, window=0, ld_extra=0, q_scale=1.0, hide=None,
                    width_extra=1):
    need = [-(-c // page) for c in ctx]
    n_pages = sum(need) + 2
    pages, at = rng.permutation(n_pages), 0
    table = np.full((len(ctx), max(need) + width_extra), -1)
    for i, k in enumerate(need):
        table[i, :k] = pages[at:at + k][:table.shape[1]]
        at += k
    if hide is not None:
        for i, j, entry in hide:
            table[i, j] = entry
    cache = make_cache(rng, n_pages, heads, page, dim)
    start = np.concatenate([[0], np.cumsum(new)])
    q = torch.from_numpy(rng.standard_normal((int(start[-1]), heads * group, dim)).astype(np.float32) * q_scale).to(TYPES[kind][1])
    scale = dim ** -0.5
    out, lse = run_attention(cache, q, kind, start, ctx, table, scale, causal, window, ld_extra)
    want, want_lse, tol, lse_tol = plain_attention(cache, q.double().numpy(), start, ctx, table, scale, causal, window)
    assert np.isfinite(out).all()
    assert (np.abs(out - want) <= tol + TYPES[kind][2] * np.abs(want) + 2.0 ** -25).all(), np.max(np.abs(out - want) - tol)
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(lse)) and (out[empty] == 0).all()
    assert (np.abs(lse[~empty] - want_lse[~empty]) <= lse_tol[~empty]).all()
    again, _ = run_attention(cache, q, kind, start, ctx, table, scale, causal, window, ld_extra, with_lse=False)
    assert np.array_equal(out, again)  # the order of the sums is fixed


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("heads,group,page", [(1, 1, 16), (8, 4, 16), (2, 8, 64), (1, 16, 32), (2, 5, 256), (3, 3, 128)])
def test_attention_of_single_tokens(kind, dim, heads, group, page):
    rng = np.random.default_rng(dim + heads * group + page)
    ctx = [1, 2, 15, 16, 17, 63, 64, 65, 700, 129]
    check_attention(rng, heads, group, dim, page, kind, [1] * len(ctx), ctx)


@pytest.mark.parametrize("kind,dim,heads,group,page", [("f16", 128, 2, 4, 16), ("bf16", 128, 1, 1, 64), ("bf16", 64, 2, 5, 32),
                                                       ("f16", 256, 1, 2, 16), ("f16", 64, 1, 16, 128), ("bf16", 256, 1, 3, 256)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 7), (True, 100), (False, 0)])
def test_attention_of_several_tokens(kind, dim, heads, group, page, causal, window):
    rng = np.random.default_rng(dim + heads * group + page + window)
    new = [1, 0, 2, 33, 5, 130, 0, 64]
    ctx = [40, 9, 2, 33, 300, 131, 0, 333]
    check_attention(rng, heads, group, dim, page, kind, new, ctx, causal, window, ld_extra=8)


# A table that could hold long requests, and many queries: what the library takes for prompts.
PROMPT = 40000


@pytest.mark.parametrize("kind,dim,heads,group,page", [("f16", 128, 2, 4, 16), ("bf16", 128, 1, 1, 64), ("bf16", 64, 2, 5, 32), ("f16", 64, 1, 16, 128),
                                                       ("bf16", 128, 1, 8, 256), ("f16", 256, 1, 2, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 3), (True, 100), (False, 0)])
def test_attention_of_prompts(kind, dim, heads, group, page, causal, window):
    rng = np.random.default_rng(dim + heads * group + page + window)
    new = [100, 0, 1, 129, 64, 0, 300, 2]
    ctx = [100, 9, 1, 200, 700, 0, 301, 128]
    check_attention(rng, heads, group, dim, page, kind, new, ctx, causal, window, ld_extra=8, width_extra=PROMPT // page)


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_of_prompts_whose_rows_see_nothing_and_pages_that_are_gone(dim):
    rng = np.random.default_rng(12)
    check_attention(rng, 2, 4, dim, 16, "bf16", [70, 40, 64, 130], [3, 0, 640, 257], width_extra=PROMPT,
                    hide=[(2, 1, -1), (2, 7, 10 ** 9), (2, 20, -7), (3, 0, -1), (3, 16, -1)])


@pytest.mark.parametrize("kind,q_scale", [("bf16", 1e-30), ("bf16", 1e4), ("f16", 1e-3), ("f16", 30.0), ("bf16", 0.0)])
def test_attention_of_prompts_of_small_and_large_queries(kind, q_scale):
    rng = np.random.default_rng(5)
    check_attention(rng, 2, 4, 128, 16, kind, [100, 30], [300, 90], q_scale=q_scale, width_extra=PROMPT)


def test_attention_of_prompts_with_scales_far_apart():
    """Value scales over 12 orders of magnitude and scales of 0: the tolerance follows the weighted magnitudes."""
    rng = np.random.default_rng(8)
    cache = list(make_cache(rng, 40, 2, 16, 128))
    cache[3] *= (10.0 ** rng.integers(-6, 7, cache[3].shape)).astype(np.float32)
    for at in ((3, 0), (7, 1), (11, 0), (12, 0), (13, 0)):
        cache[3][at] = 0.0
        cache[1][at] = 0
    cache[2][5, 0] = 0.0
    cache[0][5, 0] = 0
    start, ctx, table = [0, 200], [640], np.concatenate([rng.permutation(40), -np.ones(4000, int)])[None]
    q = torch.from_numpy(rng.standard_normal((200, 4, 128)).astype(np.float32)).to(torch.bfloat16)
    for rows in (q, q[:3]):  # the kernel for prompts and the one for few rows
        start[1] = len(rows)
        out, lse = run_attention(cache, rows, "bf16", start, ctx, table, 0.09)
        want, want_lse, tol, lse_tol = plain_attention(cache, rows.double().numpy(), start, ctx, table, 0.09, True, 0)
        assert (np.abs(out - want) <= tol + 2.0 ** -8 * np.abs(want)).all() and (np.abs(lse - want_lse) <= lse_tol).all()


def test_attention_rows_that_see_nothing_and_pages_that_are_gone():
    rng = np.random.default_rng(11)
    # more queries than tokens (the first ones stand before the first token), an empty cache, hidden pages
    check_attention(rng, 2, 4, 128, 16, "bf16", [5, 1, 1, 3, 1], [3, 0, 40, 64, 16],
                    hide=[(2, 1, -1), (3, 0, 10 ** 9), (3, 2, -7), (4, 0, -1)])
    # a table row that is shorter than the request
    check_attention(rng, 1, 2, 64, 16, "f16", [1, 4], [100, 90], width_extra=-2)


@pytest.mark.parametrize("kind,q_scale", [("bf16", 1e-30), ("bf16", 1e4), ("f16", 1e-3), ("f16", 30.0), ("bf16", 0.0)])
def test_attention_of_small_and_large_queries(kind, q_scale):
    rng = np.random.default_rng(5)
    check_attention(rng, 2, 4, 128, 16, kind, [1, 3], [200, 90], q_scale=q_scale)


def test_attention_garbage_behind_the_last_token_does_not_count():
    rng = np.random.default_rng(6)
    cache = list(make_cache(rng, 4, 1, 64, 64))
    table, q = np.array([[2, 1]]), torch.from_numpy(rng.standard_normal((1, 2, 64)).astype(np.float32)).to(torch.float16)
    cache[2][1] = cache[3][1] = np.nan  # a page that holds none of the request's tokens yet
    a, la = run_attention(cache, q, "f16", [0, 1], [50], table, 0.1)
    cache[0][2, :, 50:] = cache[1][2, :, 50:] = 127
    c, lc = run_attention(cache, q, "f16", [0, 1], [50], table, 0.1)
    assert np.isfinite(a).all() and np.array_equal(a, c) and np.array_equal(la, lc)


@pytest.mark.parametrize("B", [130, 300])
def test_attention_of_many_requests(B):
    rng = np.random.default_rng(B)
    check_attention(rng, 1, 2, 64, 16, "bf16", rng.integers(0, 4, B).tolist(), rng.integers(3, 90, B).tolist())


def test_attention_of_a_long_request():
    """One request over all blocks: 40,000 tokens of ragged pages."""
    rng = np.random.default_rng(9)
    check_attention(rng, 1, 4, 128, 16, "f16", [1, 2], [40000, 17])


def test_cache_whose_offsets_pass_32_bits():
    """A pool of over 2^32 bytes of keys: its last pages are written and read."""
    heads, dim, page = 2, 256, 256
    n_pages = 2 ** 32 // (heads * dim * page) + 8
    k, v = (torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((n_pages, heads), device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    T = 2 * page
    x = torch.empty((T, 2, heads, dim), device="cuda").normal_(generator=g).to(torch.float16)
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device="cuda")
    slots = (table[0].long()[:, None] * page + torch.arange(page, device="cuda")).reshape(-1)
    c = b.kv_cache(k, v, ks, vs, n_pages, heads, page, dim)
    b.awe_kv_write(handle(), c, x, x[:, 1], b.F16, T, 2 * heads * dim, 2 * heads * dim, slots)
    q = torch.empty((1, heads, dim), device="cuda").normal_(generator=g).to(torch.float16)
    out = torch.empty_like(q)
    work = torch.empty(b.awe_kv_attention_workspace_bytes(handle(), c, 1, heads, 1), dtype=torch.uint8, device="cuda")
    one = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    b.awe_kv_attention(handle(), c, q, b.F16, 1, heads, heads * dim, one, torch.tensor([T], dtype=torch.int32, device="cuda"), 1, table, 2,
                       2, dim ** -0.5, True, 0, out, heads * dim, None, work)
    p = table[0].long().cpu()
    small = [t[p].cpu().numpy() for t in (k, v, ks, vs)]
    want, _, tol, _ = plain_attention(small, q.double().cpu().numpy(), [0, 1], [T], np.array([[0, 1]]), dim ** -0.5, True, 0)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol + 2.0 ** -11 * np.abs(want)).all()
    used = torch.zeros(n_pages, dtype=torch.bool)
    used[p] = True
    assert int((ks.cpu()[~used] != 0).sum()) == 0 and int(k[:n_pages - 3].view(torch.int64).ne(0).sum()) == 0


# ------------------------------------------------------------------ streams, graphs, refusals
def test_a_step_on_another_stream_and_in_a_graph():
    """plan -> write -> attention, on a side stream and replayed with other lengths; nothing waits on the host."""
    rng = np.random.default_rng(2)
    heads, group, dim, page, B = 2, 4, 128, 16, 3
    n_pages, width = 40, 8
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.zeros((n_pages, heads, page, dim), dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((n_pages, heads), device="cuda") for _ in range(2))
    c = b.kv_cache(k, v, ks, vs, n_pages, heads, page, dim)
    i32 = dict(dtype=torch.int32, device="cuda")
    most = 16
    cached, new = torch.zeros(B, **i32), torch.tensor([5, 6, 5], **i32)
    table, free = torch.full((B, width), -1, **i32), torch.from_numpy(rng.permutation(n_pages).astype(np.int32)).cuda()
    slots, start, ctx, counts = torch.empty(most, dtype=torch.int64, device="cuda"), torch.empty(B + 1, **i32), torch.empty(B, **i32), torch.empty(4, **i32)
    x = torch.empty((most, (group + 2) * heads, dim), device="cuda").normal_(generator=g).to(torch.bfloat16)
    out = torch.zeros((most, heads * group, dim), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(b.awe_kv_attention_workspace_bytes(handle(), c, most, heads * group, B), dtype=torch.uint8, device="cuda")
    ld = (group + 2) * heads * dim

    def step(stream):
        b.awe_kv_plan(handle(), cached, new, B, page, free, n_pages, table, width, width, slots, None, most, start, ctx, counts, stream=stream)
        b.awe_kv_write(handle(), c, x[:, group * heads:], x[:, (group + 1) * heads:], b.BF16, most, ld, ld, slots, stream=stream)
        b.awe_kv_attention(handle(), c, x, b.BF16, most, heads * group, ld, start, ctx, B, table, width, width, dim ** -0.5, True, 0, out,
                           heads * group * dim, None, work, stream=stream)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    launches = b.awe_launch_count(handle())
    step(side)
    assert b.awe_launch_count(handle()) > launches
    side.synchronize()

    def check():
        n = int(start[-1])
        cache = [t.cpu().numpy() for t in (k, v, ks, vs)]
        want, _, tol, _ = plain_attention(cache, x[:, :group * heads].double().cpu().numpy(), start.cpu().numpy(), ctx.cpu().numpy(),
                                          table.cpu().numpy(), dim ** -0.5, True, 0)
        got = out.double().cpu().numpy()
        assert (np.abs(got - want)[:n] <= (tol + 2.0 ** -8 * np.abs(want))[:n]).all()

    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream())
    for lengths in ([1, 1, 1], [9, 0, 7], [0, 16, 0]):
        cached.copy_(ctx)
        free.copy_(torch.roll(free, -int(counts[0])))
        new.copy_(torch.tensor(lengths, **i32))
        graph.replay()
        torch.cuda.synchronize()
        assert ctx.tolist() == [c0 + n for c0, n in zip(cached.tolist(), lengths)]
        check()


def test_refusals():
    INVALID, UNSUPPORTED, WORKSPACE, ALIGNMENT = 1, 2, 3, 4
    h = handle()
    d = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    z = lambda **kw: b.KvCache(**{**dict(k_dev=d.data_ptr(), v_dev=d.data_ptr(), k_scale_dev=d.data_ptr(), v_scale_dev=d.data_ptr(),  # noqa: E731
                                         n_pages=2, n_heads=2, page_size=16, head_dim=64), **kw})
    at = d.data_ptr()
    null = ctypes.c_void_p()

    def attn(cache=None, h_=h, q=at, dt=b.F16, T=1, Hq=4, ldq=256, start=at, ctx=at, B=1, table=at, width=1, ldt=1, causal=1, window=0, out=at,
             ldo=256, lse=0, work=at, size=1 << 40):
        return b.lib().awe_kv_attention(h_ if h_ is null else h_.raw, cache if cache is not None else z(), q, dt, T, Hq, ldq, start, ctx, B, table,
                                        width, ldt, 1.0, causal, window, out, ldo, lse, work, size, None)

    launches = b.awe_launch_count(h)
    assert attn(h_=null) == INVALID
    for bad in (dict(q=0), dict(start=0), dict(ctx=0), dict(table=0), dict(out=0), dict(work=0), dict(T=-1), dict(B=-1), dict(Hq=3), dict(Hq=0),
                dict(width=0), dict(ldt=0), dict(window=-1), dict(window=3, causal=0), dict(dt=9), dict(T=2, ldq=8), dict(T=2, ldo=8),
                dict(cache=z(k_dev=0)), dict(cache=z(v_scale_dev=0)), dict(cache=z(n_pages=0)), dict(cache=z(n_heads=-1))):
        assert attn(**bad) == INVALID, bad
    for bad in (dict(dt=b.F32), dict(cache=z(page_size=24)), dict(cache=z(page_size=8)), dict(cache=z(page_size=512)), dict(cache=z(head_dim=96)),
                dict(B=b.KV_MAX_REQUESTS + 1)):
        assert attn(**bad) == UNSUPPORTED, bad
    for bad in (dict(q=at + 2), dict(out=at + 8), dict(ldq=260), dict(ldo=258), dict(work=at + 16), dict(lse=at + 2), dict(start=at + 1),
                dict(cache=z(k_dev=at + 8))):
        assert attn(**bad) == ALIGNMENT, bad
    assert attn(size=64) == WORKSPACE
    assert attn(T=0, q=0) == 0 and attn(B=0) == 0  # an empty batch
    assert b.awe_kv_attention_workspace_bytes(h, z(head_dim=80), 1, 4, 1) == 0

    def write(cache=None, k=at, v=at, dt=b.F16, T=2, ldk=128, ldv=128, slots=at):
        return b.lib().awe_kv_write(h.raw, cache if cache is not None else z(), k, v, dt, T, ldk, ldv, slots, None)

    for bad in (dict(k=0), dict(v=0), dict(slots=0), dict(T=-1), dict(ldk=100), dict(ldv=0), dict(dt=7)):
        assert write(**bad) == INVALID, bad
    assert write(dt=b.F32) == UNSUPPORTED and write(k=at + 1) == ALIGNMENT and write(slots=at + 4) == ALIGNMENT and write(T=0, k=0) == 0

    def plan(cached=at, new=at, B=1, page=16, free=at, n_free=1, table=at, width=1, ldt=1, slots=at, positions=0, most=1, start=at, ctx=at, counts=at):
        return b.lib().awe_kv_plan(h.raw, cached, new, B, page, free, n_free, table, width, ldt, slots, positions, most, start, ctx, counts, None)

    for bad in (dict(cached=0), dict(new=0), dict(B=-1), dict(free=0), dict(n_free=-1), dict(table=0), dict(width=0), dict(ldt=0), dict(slots=0),
                dict(most=-1), dict(start=0), dict(ctx=0), dict(counts=0)):
        assert plan(**bad) == INVALID, bad
    for bad in (dict(page=17), dict(page=8), dict(page=1024), dict(B=b.KV_MAX_REQUESTS + 1)):
        assert plan(**bad) == UNSUPPORTED, bad
    assert plan(slots=at + 4) == ALIGNMENT and plan(table=at + 2) == ALIGNMENT
    assert b.awe_launch_count(h) == launches  # nothing was enqueued
