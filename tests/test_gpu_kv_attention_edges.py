"""Attention over the 8-bit cache where it can go wrong: scales of 0, windows over prompts, places that nothing may read.

The reference is the definition in 64 bits.  Tolerance, with u the unit roundoff of the output type, A = sum_j p_j |v_j|, S the
largest sum of magnitudes behind a visible score and e = 2 (D / 16 + 3) 2^-22 S (FP32 sums of D / 16 matrix steps): the
softmax weights, times the values' scale in the kernel for prompts, are rounded to FP16 relative to their largest so far, which
costs 2^-11 of each or, below FP16's normal range, `floor` of the largest; each carries an integer of at most 128, so
  |out - ref| <= u |ref| + (2^-11 + e) (A + |ref|) + n floor 128 max vs,   |lse - ref| <= e + 2^-21 (1 + |ref|).
"""
import numpy as np
import pytest
import torch

from paper_2609_24519_b200 import binding as b
from tests.gpu_util import handle
from tests.test_gpu_kv_cache import TYPES, make_cache, run_attention

pytestmark = pytest.mark.gpu

WIDE = 40000  # tokens that a block table could hold: with many queries, what the library takes for prompts


def reference(cache, q, start, ctx, table, scale, causal, window):
    """out, lse, A, S, n max vs; rows that see nothing have 0, -inf, 0, 0, 0."""
    k, v, ks, vs = cache
    n_pages, heads, page, dim = k.shape
    T, Hq, _ = q.shape
    group = Hq // heads
    out, A, lse = np.zeros((T, Hq, dim)), np.zeros((T, Hq, dim)), np.full((T, Hq), -np.inf)
    S, n_vs = np.zeros((T, Hq)), np.zeros((T, Hq))
    for i, length in enumerate(ctx):
        a, n = int(start[i]), int(start[i + 1] - start[i])
        tok = np.arange(min(length, table.shape[1] * page))
        if not n or not len(tok):
            continue
        entry = table[i, tok // page]
        fine = (entry >= 0) & (entry < n_pages)
        entry = np.where(fine, entry, 0)
        place = length - n + np.arange(n)[:, None]
        seen = np.broadcast_to(fine, (n, len(tok))) & ((tok <= place) if causal else True)
        if window:
            seen = seen & (tok > place - window)
        some = seen.any(1)
        used = seen.any(0)
        for h in range(heads):
            K = k[entry, h, tok % page].astype(float) * np.where(used, ks[entry, h], 0.0)[:, None]
            V = v[entry, h, tok % page].astype(float) * np.where(used, vs[entry, h], 0.0)[:, None]
            top_vs = np.where(seen, np.where(used, vs[entry, h], 0.0), 0.0).max(1)
            for j in range(h * group, (h + 1) * group):
                x = q[a:a + n, j]
                s = np.where(seen, x @ K.T * scale, -np.inf)[some]
                m = s.max(1, keepdims=True)
                p = np.exp(s - m)
                total = p.sum(1, keepdims=True)
                rows = np.arange(a, a + n)[some]
                out[rows, j], A[rows, j] = p @ V / total, p @ np.abs(V) / total
                lse[rows, j] = (m + np.log(total))[:, 0]
                S[rows, j] = np.where(seen, np.abs(x) @ np.abs(K).T * abs(scale), 0.0).max(1)[some]
                n_vs[rows, j] = (seen.sum(1) * top_vs)[some]
    return out, lse, A, S, n_vs


def check(cache, q, kind, start, ctx, table, scale, causal=True, window=0, prompts=None, floor=2.0 ** -25):
    """Compares one call with the reference; prompts: which kernel it has to be (three launches, or at most two)."""
    launches = b.awe_launch_count(handle())
    out, lse = run_attention(cache, q, kind, start, ctx, table, scale, causal, window)
    launches = b.awe_launch_count(handle()) - launches
    assert prompts is None or (launches == 3) == prompts
    want, want_lse, A, S, n_vs = reference(cache, q.double().numpy(), start, ctx, table, scale, causal, window)
    e = 2 * (q.shape[2] / 16 + 3) * 2.0 ** -22 * S
    u = TYPES[kind][2]
    tol = u * np.abs(want) + (2.0 ** -11 + e[..., None]) * (A + np.abs(want)) + (floor * 128 * n_vs)[..., None]
    tol += 2.0 ** -25 if kind == "f16" else 1e-38  # the smallest steps of the output type
    assert np.isfinite(out).all()
    assert (np.abs(out - want) <= tol).all(), float(np.max(np.abs(out - want) / tol))
    empty = np.isneginf(want_lse)
    assert np.array_equal(empty, np.isneginf(lse)) and (out[empty] == 0).all()
    lse, want_lse, e = lse[~empty], want_lse[~empty], e[~empty]
    assert (np.abs(lse - want_lse) <= e + 2.0 ** -21 * (1 + np.abs(want_lse))).all()
    return out, lse


def normal(rng, *shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32))


def one_request(rng, n_pages, page=16):
    """A shuffled table of one request over the whole pool, as wide as WIDE tokens."""
    return np.concatenate([rng.permutation(n_pages), np.full(WIDE // page, -1)])[None]


# ------------------------------------------------------------------ value scales of 0
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("rows", [200, 3])  # the kernel for prompts, the one for few rows
def test_a_page_of_value_scale_0_counts_as_zeros_whatever_its_bytes(dim, rows):
    rng = np.random.default_rng(dim + rows)
    cache = make_cache(rng, 40, 2, 16, dim)
    cache[3][rng.random((40, 2)) < 0.3] = 0.0  # their bytes stay
    q = normal(rng, rows, 8 if dim == 64 else 4, dim).to(torch.bfloat16)
    check(cache, q, "bf16", [0, rows], [633], one_request(rng, 40), dim ** -0.5, prompts=rows == 200)


@pytest.mark.parametrize("vs", [0.02, 1e-6, 1e-9, 3e4])
@pytest.mark.parametrize("zero", ["before", "behind", "between", "odd pages"])
@pytest.mark.parametrize("rows", [300, 2])
def test_whole_steps_of_value_scale_0(vs, zero, rows):
    """Tokens without values weigh in the divisor alone, and take no bits from the others."""
    rng = np.random.default_rng(7)
    cache = make_cache(rng, 40, 1, 16, 128)
    cache[3][:] *= vs / 0.02
    table = one_request(rng, 40)
    at = np.arange(40)
    off = {"before": at < 16, "behind": at >= 16, "between": (at >= 8) & (at < 24), "odd pages": at % 2 == 1}[zero]
    cache[3][table[0, :40][off]] = 0.0
    q = normal(rng, rows, 4, 128).to(torch.bfloat16)
    check(cache, q, "bf16", [0, rows], [640], table, 0.3, prompts=rows == 300)


@pytest.mark.parametrize("rows", [200, 2])
def test_nothing_but_value_scales_of_0(rows):
    rng = np.random.default_rng(9)
    cache = make_cache(rng, 40, 2, 16, 128)
    cache[3][:] = 0.0
    out, _ = check(cache, normal(rng, rows, 4, 128).to(torch.float16), "f16", [0, rows], [630], one_request(rng, 40), 0.1, prompts=rows == 200)
    assert (out == 0).all()


@pytest.mark.parametrize("vs", [2.0 ** -106, 2.0 ** 90])
@pytest.mark.parametrize("rows", [200, 2])
def test_the_smallest_and_the_largest_value_scales(vs, rows):
    """What the cache write stores of BF16 values from 2^-99, about the least that counts for a scale, to 2^97."""
    rng = np.random.default_rng(10)
    cache = make_cache(rng, 40, 2, 16, 128)
    cache[3][:] = np.float32(vs)
    check(cache, normal(rng, rows, 4, 128).to(torch.bfloat16), "bf16", [0, rows], [640], one_request(rng, 40), 0.1, prompts=rows == 200)


# ------------------------------------------------------------------ windows over prompts
@pytest.mark.parametrize("kind,dim,heads,group,page,new,ctx", [
    ("bf16", 128, 8, 4, 16, [300, 129, 64], [700, 129, 411]), ("f16", 128, 2, 16, 64, [257, 300, 1], [257, 1500, 900]),
    ("bf16", 64, 8, 4, 32, [500, 300], [513, 1111]), ("f16", 64, 4, 5, 256, [900, 200], [900, 300]), ("f16", 128, 1, 1, 128, [5000], [5003])])
@pytest.mark.parametrize("window", [1, 3, 100, 128, 1000])
def test_prompts_under_a_window(kind, dim, heads, group, page, new, ctx, window):
    rng = np.random.default_rng(dim + heads * group + page + window)
    need = [-(-c // page) for c in ctx]
    pages, at = rng.permutation(sum(need) + 2), 0
    table = np.full((len(ctx), max(need) + WIDE // page), -1)
    for i, n in enumerate(need):
        table[i, :n] = pages[at:at + n]
        at += n
    cache = make_cache(rng, sum(need) + 2, heads, page, dim)
    q = normal(rng, sum(new), heads * group, dim).to(TYPES[kind][1])
    check(cache, q, kind, np.concatenate([[0], np.cumsum(new)]), ctx, table, dim ** -0.5, window=window, prompts=True)


# ------------------------------------------------------------------ places that no row sees
@pytest.mark.parametrize("bad", [np.nan, np.inf])
@pytest.mark.parametrize("rows,ctx", [(1, 700), (5, 700), (300, 700), (700, 1500)])  # the last is enough for the kernel for prompts
@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_pages_in_front_of_the_window_are_not_followed(bad, rows, ctx, kind):
    """Their entries may name a page that has been given up since, whatever its scales are now."""
    rng = np.random.default_rng(rows)
    n_pages, window = -(-ctx // 16) + 2, 100
    cache = make_cache(rng, n_pages, 2, 16, 128)
    cache[2][-1] = cache[3][-1] = bad
    table = one_request(rng, n_pages - 1)
    table[0, :(ctx - rows + 1 - window) // 16] = n_pages - 1  # the pages in front of the first row's first token
    check(cache, normal(rng, rows, 8, 128).to(TYPES[kind][1]), kind, [0, rows], [ctx], table, 0.09, window=window, prompts=rows == 700)


@pytest.mark.parametrize("rows", [6, 300])
def test_pages_behind_the_last_row_of_the_call_are_not_followed(rows):
    """Rows that stand in front of the first token see nothing, and make no page visible."""
    rng = np.random.default_rng(rows)
    cache = make_cache(rng, 6, 1, 16, 128)
    cache[2][5] = cache[3][5] = np.nan
    table = np.full((2, WIDE // 16), 5)
    table[0, :2], table[1, :3] = [1, 2], [0, 3, 4]
    # 20 and 48 tokens; the entries behind them name the bad page
    check(cache, normal(rng, 2 * rows, 8, 128).to(torch.bfloat16), "bf16", [0, rows, 2 * rows], [20, 48], table, 0.09, prompts=rows == 300)


# ------------------------------------------------------------------ range of the weights and of the queries
FLOOR = 2.0 ** -35  # of the largest weight: what a rounded weight may be off by where it is far below


@pytest.mark.parametrize("lead", [20, 24, 26])
@pytest.mark.parametrize("tokens,rows", [(256, 1), (8192, 1), (8192, 200)])
@pytest.mark.parametrize("leader", ["first", "last"])
def test_a_token_without_values_that_leads_the_others_far(lead, tokens, rows, leader):
    """The others' weights are 2^-lead of the leader's, and they alone make the result."""
    rng = np.random.default_rng(lead)
    dim, page, n_pages = 128, 16, tokens // 16
    cache = make_cache(rng, n_pages, 1, page, dim)
    cache[0][:], cache[2][:], cache[3][:] = 100, np.float32(0.01), np.float32(0.02)
    cache[1][:] = rng.integers(1, 128, cache[1].shape)
    at = (0, 0) if leader == "first" else (n_pages - 1, page - 1)
    cache[0][at[0], 0, at[1]], cache[1][at[0], 0, at[1]] = 120, 0
    q = torch.ones((rows, 2, dim)).to(torch.float16)
    scale = lead * np.log(2) / (20 * dim * 0.01)
    table = np.concatenate([np.arange(n_pages), np.full(0 if tokens == 256 else WIDE // page, -1)])[None]
    check(cache, q, "f16", [0, rows], [tokens], table, scale, causal=False, prompts=rows == 200, floor=FLOOR)


@pytest.mark.parametrize("rows", [200, 3])
@pytest.mark.parametrize("dim", [64, 128])
def test_bf16_queries_with_one_element_far_above_the_others(rows, dim):
    """Keys are 0 there, so the small elements alone make the scores."""
    rng = np.random.default_rng(dim)
    cache = make_cache(rng, 40, 2, 16, dim)
    cache[0][..., 5] = 0
    q = normal(rng, rows, 8, dim)
    q[..., 5] = 2.0 ** 21
    q[1, 0, 5], q[2, 0, 5] = -2.0 ** 20, 2.0 ** -10
    q[0, 0], q[0, 0, 5] = 0.0, 2.0 ** 127  # by itself: scores of 0
    check(cache, q.to(torch.bfloat16), "bf16", [0, rows], [640], one_request(rng, 40), dim ** -0.5, prompts=rows == 200, floor=FLOOR)


@pytest.mark.parametrize("rows", [200, 3])
@pytest.mark.parametrize("q_scale", [2.0 ** -126, 2.0 ** -115, 2.0 ** 60])
def test_bf16_queries_at_the_ends_of_their_range(rows, q_scale):
    rng = np.random.default_rng(4)
    cache = make_cache(rng, 40, 2, 16, 128)
    q = (normal(rng, rows, 8, 128) * q_scale).to(torch.bfloat16)
    scale = float(np.float32(0.09 / max(q_scale, 2.0 ** -60)))
    check(cache, q, "bf16", [0, rows], [640], one_request(rng, 40), scale, prompts=rows == 200, floor=FLOOR)


# ------------------------------------------------------------------ many requests of short contexts
@pytest.mark.parametrize("B,launches", [(100, 1), (2048, 2)])
def test_short_contexts_of_many_requests(B, launches):
    """A block per unit, each of which scans the requests, where those are few; else the units in parts."""
    rng = np.random.default_rng(B)
    ctx = rng.integers(0, 40, B).tolist()
    cache = make_cache(rng, 500, 2, 16, 64)
    table = rng.integers(0, 500, (B, 3))
    q = normal(rng, B, 2, 64).to(torch.bfloat16)
    before = b.awe_launch_count(handle())
    check(cache, q, "bf16", np.arange(B + 1), ctx, table, 0.125, floor=FLOOR)
    assert b.awe_launch_count(handle()) - before == launches
