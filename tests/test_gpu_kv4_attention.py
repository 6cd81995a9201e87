"""awe_kv4_attention against softmax attention in 64 bits over the values that the 4-bit cache's bytes stand for.

Tolerance.  A score's sum of D exact products is off by at most D 2^-23 of the sum of their magnitudes, the exponential and the rest of
its argument by 2^-20 of the weight; a weight is rounded to FP16 by 2^-11 of itself, or by 2^-35 of the largest contribution (weight times
scale, codes up to 15); the output by eps / 2.  BF16 queries keep all bits down to 2^-32 of their row's largest."""
import math

import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle

pytestmark = pytest.mark.gpu
TORCH = {b.F16: torch.float16, b.BF16: torch.bfloat16}


def make(new, ctx, Hq, H, D, page, dtype, window=0, causal=True, seed=0, pad=0, scales=None, width=None, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, T = len(new), sum(new)
    want = [-(-c // page) for c in ctx]
    width = width or max(max(want), 1) + 1
    pool = sum(want) + 2
    order = torch.randperm(pool, generator=g, device="cuda").to(torch.int32).tolist()
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(want):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    u8 = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731

    def params():
        lo, hi = scales or (0.02, 0.6)
        s = torch.rand((pool, H, page), generator=g, device="cuda").mul_(math.log2(hi / lo)).add_(math.log2(lo)).exp2_()
        zero = torch.randint(0, 16, s.shape, generator=g, device="cuda", dtype=torch.int16)
        return ((s * 16).half().view(torch.int16) & -16) | zero

    start = [0]
    for n in new:
        start.append(start[-1] + n)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.empty((T, Hq * D + pad), device="cuda").normal_(0.0, spread, generator=g).to(TORCH[dtype])
    return dict(B=B, T=T, Hq=Hq, H=H, D=D, page=page, dtype=dtype, window=window, causal=causal, new=new, ctx=ctx, pool=pool, width=width,
                table=table.cuda(), k=u8(pool, H, page, D // 2), v=u8(pool, H, page, D // 2), kp=params(), vp=params(), q=q, start=ints(start),
                ctx_len=ints(ctx), scale=D ** -0.5, out=torch.full((T + 2, Hq * D + pad), 7.0, device="cuda", dtype=TORCH[dtype]),
                lse=torch.full((T + 2, Hq), 7.0, device="cuda"))


def call(s, workspace=None):
    cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], s["H"], s["page"], s["D"])
    if workspace is None:
        n = b.awe_kv4_attention_workspace_bytes(handle(), cache, s["T"], s["Hq"], s["B"])
        workspace = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    before = b.awe_launch_count(handle())
    b.awe_kv4_attention(handle(), cache, s["q"], s["dtype"], s["T"], s["Hq"], s["q"].stride(0), s["start"], s["ctx_len"], s["B"], s["table"], s["width"],
                        s["width"], s["scale"], s["causal"], s["window"], s["out"], s["out"].stride(0), s["lse"], workspace)
    return b.awe_launch_count(handle()) - before


def values(codes, par):
    """scale * (code - zero) in 64 bits; scales within the format's bounds."""
    c, p = codes.to(torch.int32), par.to(torch.int32) & 0xFFFF
    x = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    signed = lambda v: ((v & 15) ^ 8) - 8  # noqa: E731
    scale = torch.nan_to_num((p & 0xFFF0).to(torch.int16).view(torch.float16).double() / 16, 2.0 ** -18).clamp(2.0 ** -18, 4064.0)
    return (signed(x) - signed(p)[..., None]).double() * scale[..., None]


def check(s):
    G, D, eps = s["Hq"] // s["H"], s["D"], torch.finfo(TORCH[s["dtype"]]).eps / 2
    q = s["q"][:, :s["Hq"] * D].double().view(s["T"], s["Hq"], D)
    got = s["out"][:s["T"], :s["Hq"] * D].double().view(s["T"], s["Hq"], D)
    at = 0
    for i, (n, c) in enumerate(zip(s["new"], s["ctx"])):
        if n == 0:
            continue
        rows = slice(at, at + n)
        at += n
        pages = s["table"][i, :-(-c // s["page"])].long()
        held = ((pages >= 0) & (pages < s["pool"])).repeat_interleave(s["page"])[:c]
        pages = pages.clamp(0, s["pool"] - 1)
        tok, pos = torch.arange(c, device="cuda"), torch.arange(c - n, c, device="cuda")[:, None]
        seen = held & (tok <= pos if s["causal"] else torch.ones((n, 1), dtype=torch.bool, device="cuda"))
        if s["window"]:
            seen = seen & (tok > pos - s["window"])
        for h in range(s["H"]):
            k = values(s["k"][pages, h], s["kp"][pages, h]).reshape(-1, D)[:c]
            v = values(s["v"][pages, h], s["vp"][pages, h]).reshape(-1, D)[:c]
            x = torch.einsum("nhd,cd->nhc", q[rows, h * G:(h + 1) * G], k) * s["scale"]
            size = torch.einsum("nhd,cd->nhc", q[rows, h * G:(h + 1) * G].abs(), k.abs()) * abs(s["scale"])
            x = x.masked_fill(~seen[:, None], -math.inf)
            lse = torch.logsumexp(x, -1) if c else torch.full((n, G), -math.inf, device="cuda", dtype=torch.float64)
            p = torch.where(lse[..., None] > -math.inf, torch.exp(x - lse[..., None]), 0.0)
            off = D * 2.0 ** -23 * size.masked_fill(~seen[:, None], 0.0).amax(-1) + 2.0 ** -20 if c else torch.zeros_like(lse)
            want, weight = p @ v, p @ v.abs()
            most = (p * v.abs().amax(-1)).amax(-1) if c else torch.zeros_like(lse)
            slack = (2.0 ** -10 + 3 * off)[..., None] * weight + (2.0 ** -30 * c * most)[..., None]
            o = got[rows, h * G:(h + 1) * G]
            assert bool(((o - want).abs() <= slack + eps * (want.abs() + slack) + 2.0 ** -25).all()), (i, h, ((o - want).abs() - slack).max())
            l = s["lse"][rows, h * G:(h + 1) * G].double()
            empty = lse == -math.inf
            assert torch.equal(l == -math.inf, empty) and bool((o[empty] == 0).all())
            assert bool(((l - lse).abs() <= 2 * off + 2.0 ** -22 * (1 + lse.abs()))[~empty].all())
    assert bool((s["out"][s["T"]:] == 7.0).all()) and bool((s["lse"][s["T"]:] == 7.0).all()) and bool((s["out"][:, s["Hq"] * D:] == 7.0).all())


FEW, TC = (1, 2), (3,)  # launches of the kernel for few rows (short contexts, others) and of that for prompts


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,H,page", [(1, 1, 16), (8, 8, 32), (32, 8, 16), (10, 2, 64), (48, 2, 256)])
def test_single_tokens(Hq, H, page, D, dtype):
    s = make([1] * 6, [1, 15, 16, 17, 300, 1000], Hq, H, D, page, dtype, seed=D + Hq)
    assert call(s) in FEW
    check(s)


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("lengths", [[1], [2], [31], [64], [65], [200, 0, 1], [0, 0, 9]])
def test_short_contexts(lengths, D):
    s = make([min(1, n) for n in lengths], lengths, 4, 2, D, 16, b.BF16, seed=sum(lengths))
    assert call(s) in FEW
    check(s)


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("window,causal", [(0, True), (1, True), (40, True), (100000, True), (0, False)])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_several_queries_windows_and_all_tokens(D, window, causal, dtype):
    s = make([5, 1, 0, 12, 3], [400, 1, 77, 12, 2], 6, 2, D, 32, dtype, window, causal, seed=window)
    assert call(s) in FEW
    check(s)


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("window,causal", [(0, True), (100, True), (1000, True), (0, False)])
@pytest.mark.parametrize("D,Hq,H,page,new,ctx", [
    (128, 8, 2, 16, [600], [1500]), (128, 8, 8, 64, [300, 257, 1], [300, 2000, 900]), (64, 16, 4, 32, [500, 33], [1100, 1000]),
    (128, 5, 1, 256, [700], [1023]), (64, 8, 8, 16, [1000], [1000])])
def test_prompts(D, Hq, H, page, new, ctx, window, causal, dtype):
    s = make(new, ctx, Hq, H, D, page, dtype, window, causal, seed=D + len(new), pad=8, width=4096 // page)
    assert call(s) in (TC if window != 100 else FEW + TC)  # of few tokens either kernel may take the call
    check(s)


def test_long_contexts():
    for D, Hq, H in ((128, 16, 2), (64, 4, 4), (256, 8, 1)):
        s = make([1, 1], [40000, 33333], Hq, H, D, 64, b.F16, seed=D)
        assert call(s) == 2
        check(s)


@pytest.mark.parametrize("D,dtype", [(64, b.F16), (128, b.BF16), (256, b.F16)])
def test_many_rows_whose_parts_are_joined(D, dtype):
    """More rows than are joined by a block each."""
    ctx = [1 + (997 * i) % 2500 for i in range(45)]
    s = make([1] * 45, ctx, 32, 4, D, 16, dtype, seed=D)
    assert call(s) == 2
    check(s)


@pytest.mark.parametrize("new,ctx", [([1, 1], [700, 64]), ([900, 40], [1000, 900])])
def test_pages_that_do_not_exist(new, ctx):
    """Entries outside the pool hide their tokens; a request with no page at all sees nothing."""
    s = make(new + [1], ctx + [50], 8, 2, 128, 16, b.F16, width=256, seed=1)
    s["table"][0, 1], s["table"][0, 3], s["table"][1, 0] = -1, s["pool"], 2 ** 31 - 1
    s["table"][2] = -5
    call(s)
    check(s)


@pytest.mark.parametrize("new,ctx", [([1], [1000]), ([900], [1000])])
@pytest.mark.parametrize("scales", [(2.0 ** -18, 2.0 ** -17), (2000.0, 4064.0), (2.0 ** -18, 4064.0)])
def test_scales_at_the_ends_of_the_range(scales, new, ctx):
    s = make(new, ctx, 8, 2, 128, 16, b.BF16, scales=scales, width=128, seed=5)
    s["kp"] = make(new, ctx, 8, 2, 128, 16, b.BF16, width=128, seed=5)["kp"]  # scores as usual
    call(s)
    check(s)


@pytest.mark.parametrize("new,ctx", [([1], [300]), ([1000], [1100])])
def test_words_that_no_append_writes(new, ctx):
    """Zeros, NaN and negative patterns are read as the format says."""
    s = make(new, ctx, 8, 2, 64, 16, b.F16, width=256, seed=6)
    for par in (s["kp"], s["vp"]):
        flat = par.view(-1)
        flat[::7], flat[1::7], flat[2::7], flat[3::7] = 0, 0x7E05, -9, 0x0013
    call(s)
    check(s)


@pytest.mark.parametrize("new,ctx", [([1, 1], [500, 20]), ([900], [1000])])
@pytest.mark.parametrize("spread", [1e-4, 40.0])
def test_flat_and_sharp_weights(spread, new, ctx):
    for dtype in (b.F16, b.BF16):
        s = make(new, ctx, 8, 2, 128, 32, dtype, width=64, spread=spread, seed=7)
        call(s)
        check(s)
        s["scale"] = -s["scale"]
        call(s)
        check(s)
        s["scale"] = 0.0
        call(s)
        check(s)


def test_requests_without_queries_and_contexts_shorter_than_the_queries():
    s = make([3, 0, 2], [5, 100, 1], 4, 4, 64, 16, b.F16, seed=3)  # the third request's first query stands before its only token
    call(s)
    check(s)


def test_context_beyond_the_table_ends_with_it():
    s = make([1], [64], 4, 1, 64, 16, b.F16, width=4)
    call(s)
    want = s["out"].clone()
    s["ctx_len"] += 1000  # non-causal: the tokens that the table has
    s["causal"] = False
    call(s)
    assert torch.equal(want, s["out"])


def test_same_bits_again_and_from_a_graph():
    for new, ctx in (([1] * 5, [300, 2000, 1, 64, 999]), ([700], [1000])):
        s = make(new, ctx, 16, 4, 128, 16, b.BF16, width=256)
        call(s)
        out, lse = s["out"].clone(), s["lse"].clone()
        call(s)
        assert torch.equal(out, s["out"]) and torch.equal(lse, s["lse"])
        cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 4, 16, 128)
        workspace = torch.zeros(b.awe_kv4_attention_workspace_bytes(handle(), cache, s["T"], 16, s["B"]), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            call(s, workspace)
        s["q"].copy_(s["q"].flip(0))
        s["ctx_len"] -= torch.tensor([max(0, c // 3 - n) for n, c in zip(new, ctx)], dtype=torch.int32, device="cuda")
        s["ctx"] = s["ctx_len"].tolist()
        graph.replay()
        torch.cuda.synchronize()
        check(s)


def test_refusals():
    s = make([1, 1], [20, 20], 4, 2, 64, 16, b.F16)
    cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 2, 16, 64)
    n = b.awe_kv4_attention_workspace_bytes(handle(), cache, 2, 4, 2)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    wide = s["q"].stride(0)

    def status(cache=cache, q=s["q"], dtype=b.F16, T=2, Hq=4, ldq=wide, start=s["start"], B=2, table=s["table"], width=s["width"], ld=s["width"], causal=True, window=0,
               out=s["out"], ldo=wide, ws=ws, size=n):
        try:
            b.awe_kv4_attention(handle(), cache, q, dtype, T, Hq, ldq, start, s["ctx_len"], B, table, width, ld, 0.1, causal, window, out, ldo, s["lse"], ws, size)
        except b.AweError as e:
            return e.status
        return b.OK

    assert status() == b.OK and status(T=0) == b.OK and status(B=0) == b.OK
    for bad in (dict(T=-1), dict(B=-1), dict(dtype=9), dict(window=-1), dict(window=4, causal=False), dict(q=None), dict(out=None), dict(start=None), dict(table=None),
                dict(ws=None), dict(Hq=0), dict(Hq=5), dict(width=0), dict(ld=s["width"] - 1), dict(ldq=248), dict(ldo=248)):
        assert status(**bad) == 1, bad
    for bad in (dict(dtype=b.F32), dict(B=b.KV_MAX_REQUESTS + 1), dict(width=2 ** 28, ld=2 ** 28),
                dict(cache=b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 2, 16, 32)), dict(cache=b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 2, 24, 64))):
        assert status(**bad) == 2, bad
    assert status(size=n - 1) == 3
    for bad in (dict(q=s["q"].view(-1)[1:]), dict(ldq=260), dict(ldo=260), dict(ws=ws[1:]), dict(cache=b.kv4_cache(s["k"].view(-1)[1:], s["v"], s["kp"], s["vp"], 2, 2, 16, 64))):
        assert status(**bad) == 4, bad
    assert b.awe_kv4_attention_workspace_bytes(handle(), cache, 2, 5, 2) == 0


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("ctx,window", [(1, 0), (2, 0), (1000, 1), (33, 3)])
def test_logarithms_of_few_tokens(ctx, window, D, dtype):
    """Where no sum evens errors out.  s / ln 2 - m lies between 8 and 16, where half an ulp is 2^-21; the exponential and the logarithm add
    2^-22 each, factor and score some 2^-23 of the score: together, as a root mean square, below ln 2 (2^-21 + 2^-21 of the score)."""
    s = make([1] * 24, [ctx] * 24, 10, 2, D, 16, dtype, window=window, seed=ctx + D)
    call(s)
    check(s)
    want = torch.empty((24, 10), dtype=torch.float64, device="cuda")
    for i in range(24):
        pages = s["table"][i, :-(-ctx // 16)].long()
        for h in range(2):
            k = values(s["k"][pages, h], s["kp"][pages, h]).reshape(-1, D)[:ctx][-window:]
            want[i, 5 * h:5 * h + 5] = torch.logsumexp(s["q"][i].double().view(10, D)[5 * h:5 * h + 5] @ k.t() * s["scale"], 1)
    size = lambda x: float(x.square().mean().sqrt())  # noqa: E731
    assert size(s["lse"][:24].double() - want) <= math.log(2) * 2.0 ** -21 * (1 + size(want) / math.log(2))


@pytest.mark.parametrize("D,dtype", [(64, b.F16), (128, b.BF16), (256, b.F16)])
@pytest.mark.parametrize("Hq,H", [(4, 4), (16, 4), (15, 3), (32, 2)])
@pytest.mark.parametrize("B", [1, 5, 12, 40])
def test_contexts_of_a_few_steps(B, Hq, H, D, dtype):
    """Clusters of two, four and eight blocks; requests that leave some of the blocks without a step, or all."""
    ctx = [(1000, 1, 300, 129, 777, 40, 128, 999, 513)[i % 9] for i in range(B)]
    s = make([1] * B, ctx, Hq, H, D, 32, dtype, seed=B + Hq)
    call(s)
    check(s)
    first = s["out"].clone()
    call(s)
    assert torch.equal(first, s["out"])
    s = make([3, 0, 1] * ((B + 2) // 3), [1000, 0, 640] * ((B + 2) // 3), Hq, H, D, 16, dtype, window=200 if B == 5 else 0, seed=B, pad=8)
    s["table"][0, :17] = -1  # its first blocks have nothing
    s["table"][-1] = -1
    call(s)
    check(s)


def test_short_contexts_take_one_launch():
    for B, ctx in ((1, 100), (1, 777), (4, 2000), (16, 500), (32, 1000)):
        assert call(make([1] * B, [ctx] * B, 32, 8, 128, 32, b.BF16, width=-(-ctx // 32))) == 1
    for B, ctx in ((1, 8000), (64, 1000)):
        assert call(make([1] * B, [ctx] * B, 32, 8, 128, 32, b.BF16, width=-(-ctx // 32))) == 2
