"""Attention over the 4-bit cache where it can go wrong: references of the softmax that move inside a step, scales far apart, the largest sizes.

In most the scores are built: one dimension of the keys carries them, each a value that the format holds, and the reference computes from the
stored bytes in 64 bits.  Tolerance, with u the unit roundoff of the output type, p_j the probabilities and P the largest: a weight is rounded to
FP16, the largest standing between 2^9 and 2^15, so by 2^-11 of itself, or by 2^-25 <= 2^-34 P where it is below 2^-14, which p_j >= 2^-23 P is not;
FP32 sums and exponentials add less than 2^-14 for the scores here (below 2^6, so that 2^-14 is many FP32 roundings of an exponent).  So
|out - ref| <= u |ref| + (1 + u) ((2^-11 + 2^-14) sum_j p_j |v_j| + 2^-34 P sum_small |v_j|) + 2^-25, the last for FP16's subnormals."""
import math

import numpy as np
import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle
from .test_gpu_kv4_attention import TORCH, call, make, values
from .test_gpu_kv_cache import make_cache, run_attention

pytestmark = pytest.mark.gpu
KINDS = [(64, b.F16), (128, b.BF16)]


def words(scale, zero):
    """Parameter words; scales are cut to the format's 7 significant bits."""
    bits = (scale * 16).half().view(torch.int16) & -16
    return bits | (zero.to(torch.int16) & 15)


def built(exponents, value_scales, rows, D, dtype, Hq=8, wide=True, seed=0):
    """One request whose `rows` (a factor each) last tokens ask: the score of token j and row r, as a base-2 exponent, is rows[r] exponents[j]
    (up to 7 bits), its values are random codes times value_scales[j].  wide: a table so wide that the kernel for prompts takes many rows."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, T, page = len(exponents), len(rows), 16
    pool = -(-n // page)
    x = torch.tensor(exponents, dtype=torch.float64, device="cuda")
    factor = 1.0 if dtype == b.F16 else 2.0
    k = torch.full((pool * page, D // 2), 0x88, dtype=torch.uint8, device="cuda")  # every code its zero point, -8
    k[:n, 0] = torch.where(x == 0, 0x88, 0x80).to(torch.uint8)  # of dimension 0: 8 scales above it
    k_scale = torch.full((pool * page,), 1.0, dtype=torch.float64, device="cuda")
    k_scale[:n] = torch.where(x == 0, 1.0, x.abs() / 8 / factor)
    v = torch.randint(0, 256, (pool * page, D // 2), generator=g, device="cuda", dtype=torch.uint8)
    v_scale = torch.full((pool * page,), 1.0, dtype=torch.float64, device="cuda")
    v_scale[:n] = torch.tensor(value_scales, dtype=torch.float64, device="cuda")
    minus8 = torch.full((pool * page,), -8, device="cuda")
    q = torch.zeros((T, Hq, D), dtype=TORCH[dtype], device="cuda")
    q[:, :, 0] = (torch.tensor(rows, device="cuda") * factor)[:, None].to(TORCH[dtype])
    width = max(pool, 4096 // page) if wide else pool
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :pool] = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    place = (table[0, :pool].long()[:, None] * page + torch.arange(page, device="cuda")).flatten()

    def spread(a):
        to = torch.empty_like(a)
        to[place] = a
        return to.view(pool, 1, page, *a.shape[1:])

    zero = torch.randint(-4, 4, (pool * page,), generator=g, device="cuda")
    return dict(n=n, T=T, Hq=Hq, D=D, dtype=dtype, page=page, pool=pool, width=width, table=table, q=q, k=spread(k), v=spread(v),
                kp=spread(words(k_scale, minus8)), vp=spread(words(v_scale, zero)), place=place[:n], scale=math.log(2.0))


def attend(s, causal=False):
    cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 1, s["page"], s["D"])
    ws = torch.empty(b.awe_kv4_attention_workspace_bytes(handle(), cache, s["T"], s["Hq"], 1), dtype=torch.uint8, device="cuda")
    start, ctx = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, s["T"]], [s["n"]]))
    out, lse = torch.empty_like(s["q"]), torch.empty((s["T"], s["Hq"]), device="cuda")
    before = b.awe_launch_count(handle())
    b.awe_kv4_attention(handle(), cache, s["q"], s["dtype"], s["T"], s["Hq"], s["Hq"] * s["D"], start, ctx, 1, s["table"], s["width"], s["width"], s["scale"],
                        causal, 0, out, s["Hq"] * s["D"], lse, ws)
    torch.cuda.synchronize()
    assert b.awe_last_device_status(handle()) == (0, 0)
    return out.double(), lse.double(), b.awe_launch_count(handle()) - before


def reference(s):
    """Output, lse, sum of p |v| and each row's probabilities, over all tokens."""
    k = values(s["k"].flatten(0, 2), s["kp"].flatten())[s["place"]]
    v = values(s["v"].flatten(0, 2), s["vp"].flatten())[s["place"]]
    x = torch.einsum("thd,nd->thn", s["q"].double(), k) * s["scale"]
    p = torch.softmax(x, -1)
    return p @ v, torch.logsumexp(x, -1), p @ v.abs(), p, v


def check(s, out, lse):
    want, want_lse, size, p, v = reference(s)
    u = torch.finfo(TORCH[s["dtype"]]).eps / 2
    most = p.amax(-1, keepdim=True)
    floor = 2.0 ** -34 * most * ((p < 2.0 ** -23 * most).double() @ v.abs())
    slack = u * want.abs() + (1 + u) * ((2.0 ** -11 + 2.0 ** -14) * size + floor) + 2.0 ** -25
    assert bool(((out - want).abs() <= slack).all()), float(((out - want).abs() / slack).max())
    assert bool(((lse - want_lse).abs() <= 2.0 ** -14 + 2.0 ** -22 * want_lse.abs()).all())


def steps_of(jumps, lead=128):
    """Exponents of steps of 128 tokens: `lead` tokens at 0, then each pair of `jumps` raises the first and the second half of a step."""
    e, level = [0.0] * lead, 0.0
    for j in jumps:
        level += j
        e += [level] * 64
    return e


@pytest.mark.parametrize("D,dtype", KINDS)
@pytest.mark.parametrize("slow", [None, 2, 31])
@pytest.mark.parametrize("jumps", [[7, 7], [6, 6, 6, 6], [0, 7, 7, 6], [8, 0, 6, 6]])
def test_references_that_move_in_both_halves_of_a_step(jumps, slow, D, dtype):
    """Every token contributes alike: values shrink as the scores rise, so what was stored before a reference moved has to be brought along.
    slow: every slow-th row's scores rise by an eighth of that, so that only some rows of a warp move theirs."""
    e = steps_of(jumps)
    rows = [0.125 if slow and i % slow == 0 else 1.0 for i in range(1024)]
    s = built(e, [2.0 ** (11 - x) for x in e], rows, D, dtype)
    out, lse, launches = attend(s)
    assert launches == 3
    check(s, out, lse)
    again, lse_again, _ = attend(s)
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("D,dtype", KINDS)
@pytest.mark.parametrize("first,second", [(4.75, 24.0), (4.75, 25.0), (4.75, 27.0), (0.0, 26.0), (4.75, 31.0), (4.75, 33.0)])
def test_first_half_of_a_step_beside_a_jump_of_many_powers_in_the_second(first, second, D, dtype):
    """Scores of 0, then a step whose first half passes the reference by too little to move it and whose last token moves it by 2^25 to 2^34: the
    first half's weights stay FP16 numbers beside the new largest one.  Its values are up to 2^29 times the others'.  So many rows that most blocks
    have whole units, whose first step comes before this one."""
    e = [0.0] * 128 + [first] * 64 + [0.0] * 63 + [second]
    large = [2.0 ** -17] * 128 + [4064.0] * 64 + [2.0 ** -17] * 64
    for value_scales in (large, [1.0] * 128 + [256.0] * 64 + [1.0] * 64):
        s = built(e, value_scales, [1.0] * 8192, D, dtype)
        out, lse, launches = attend(s)
        assert launches == 3
        check(s, out, lse)


@pytest.mark.parametrize("D,dtype", KINDS)
@pytest.mark.parametrize("first", [True, False])
@pytest.mark.parametrize("below", [20, 26, 33, 36, 40])
def test_token_of_least_scale_above_tokens_of_large_scale(below, first, D, dtype):
    """The dominant token contributes next to nothing.  For few rows the others count by what they contribute (their weight times scale, q_j, by
    2^-34 of the largest q: 2^-25 below 2^9); for prompts by their weight."""
    e, scales = [float(below)] + [0.0] * 300, [2.0 ** -18] + [4064.0] * 300
    if not first:
        e.reverse(), scales.reverse()
    s = built(e, scales, [1.0] * 1024, D, dtype)
    out, lse, launches = attend(s)
    assert launches == 3
    check(s, out, lse)
    for rows in ([1.0], [1.0, 0.5, 0.25]):
        s = built(e, scales, rows, D, dtype, wide=False)
        out, lse, launches = attend(s)
        assert launches < 3
        want, want_lse, size, p, v = reference(s)
        vs = torch.tensor(scales, dtype=torch.float64, device="cuda")
        q, u = p * vs, torch.finfo(TORCH[dtype]).eps / 2
        most = q.amax(-1, keepdim=True)
        floor = 2.0 ** -34 * most * ((q < 2.0 ** -23 * most).double() @ (v.abs() / vs[:, None]))
        slack = u * want.abs() + (1 + u) * ((2.0 ** -11 + 2.0 ** -14) * size + floor) + 2.0 ** -25
        assert bool(((out - want).abs() <= slack).all()), float(((out - want).abs() / slack).max())
        assert bool(((lse - want_lse).abs() <= 2.0 ** -14 + 2.0 ** -22 * want_lse.abs()).all())


@pytest.mark.parametrize("D,dtype", [*KINDS, (256, b.F16)])
@pytest.mark.parametrize("zero", [-8, 0, 7])
@pytest.mark.parametrize("other", [0, 1])
def test_keys_whose_codes_are_their_zero_point_but_for_one_channel(other, zero, D, dtype):
    """A score of few rows is the difference of sum q (code + 8) and (zero + 8) sum q, whose terms may be large where sum |q k| is small or 0.  Each is
    a sum of D / 16 matrix steps (D / 2 additions) of at most 15 sum |q| in all: off by D 2^-23 of that, times key scale and factor."""
    s = built([1.0] * 40, [1.0] * 40, [1.0], D, dtype, wide=False)
    g = torch.Generator(device="cuda").manual_seed(zero + 9)
    code = (zero & 15) * 17
    s["k"].fill_(code)
    s["k"][..., 3] = code if not other else ((zero & 15) << 4) | ((zero + (1 if zero < 7 else -1)) & 15)
    s["kp"][:] = words(torch.full_like(s["kp"], 1.0, dtype=torch.float64), torch.full_like(s["kp"], zero))
    s["q"].normal_(0.0, 4.0, generator=g)
    s["scale"] = D ** -0.5
    out, lse, _ = attend(s)
    _, want, _, _, _ = reference(s)
    q = s["q"].double().abs()
    small = D * 2.0 ** -23 * q[..., 6] * s["scale"] * other + 2.0 ** -20 * (1 + want.abs())
    bound = small + D * 2.0 ** -23 * 15 * q.sum(-1) * s["scale"]
    assert bool(((lse - want).abs() <= bound).all()), float(((lse - want).abs() / bound).max())


LONGEST = [2 ** 31 - 1, 2 ** 31, 2 ** 62, 2 ** 63 - 129, 2 ** 63 - 1]


@pytest.mark.parametrize("window", LONGEST)
@pytest.mark.parametrize("new,ctx,width", [([1, 1], [9000, 8800], 563), ([1], [777], 49), ([600], [1500], 256)])
def test_windows_longer_than_any_context(new, ctx, width, window):
    """The same kernels and bits as without a window."""
    s = make(new, ctx, 8, 2, 128, 16, b.BF16, width=width, seed=2)
    launches = call(s)
    out, lse = s["out"].clone(), s["lse"].clone()
    s["window"] = window
    assert call(s) == launches
    assert torch.equal(out, s["out"]) and torch.equal(lse, s["lse"])


@pytest.mark.parametrize("window", LONGEST)
@pytest.mark.parametrize("rows,pages", [(1, 600), (300, 40)])
def test_windows_longer_than_any_context_over_the_cache_of_8_bits(rows, pages, window):
    rng = np.random.default_rng(rows)
    cache = make_cache(rng, pages, 2, 16, 128)
    q = torch.from_numpy(rng.standard_normal((rows, 8, 128)).astype(np.float32)).to(torch.bfloat16)
    table = np.concatenate([rng.permutation(pages), np.full(0 if rows == 1 else 2000, -1)])[None]
    args = (cache, q, "bf16", [0, rows], [16 * pages - 3], table, 128 ** -0.5)
    counts = [b.awe_launch_count(handle())]
    got = []
    for w in (0, window):
        got.append(run_attention(*args, window=w))
        counts.append(b.awe_launch_count(handle()))
    assert counts[1] - counts[0] == counts[2] - counts[1] == (3 if rows > 1 else 2)
    assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])


@pytest.mark.parametrize("T", [2 ** 31, 2 ** 60, 2 ** 62 + 2, 2 ** 63 - 1])
def test_more_queries_than_32_bits_count(T):
    s = make([1], [20], 16, 2, 64, 16, b.F16)
    s["T"] = T
    cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["pool"], 2, 16, 64)
    with pytest.raises(b.AweError) as e:
        b.awe_kv4_attention(handle(), cache, s["q"], b.F16, T, 16, 1024, s["start"], s["ctx_len"], 1, s["table"], s["width"], s["width"], 0.1, True, 0, s["out"],
                            1024, s["lse"], s["k"], 2 ** 62)
    assert e.value.status == 2


def long_call(four, D, pool, table, q, new, ctx, window):
    """One request over a pool of pages of 16 tokens and one head; q: new x Hq x D BF16."""
    page, Hq = 16, q.shape[1]
    g = torch.Generator(device="cuda").manual_seed(D)
    if four:
        s = make([1], [16 * pool - 32], 1, 1, D, page, b.BF16, seed=D)
        assert s["pool"] == pool
        cache = b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], pool, 1, page, D)
        size, attention = b.awe_kv4_attention_workspace_bytes, b.awe_kv4_attention
    else:
        k, v = (torch.randint(-127, 128, (pool, 1, page, D), generator=g, device="cuda", dtype=torch.int8) for _ in range(2))
        scales = torch.full((pool, 1), 0.02, device="cuda")
        cache = b.kv_cache(k, v, scales, scales, pool, 1, page, D)
        size, attention = b.awe_kv_attention_workspace_bytes, b.awe_kv_attention
    ws = torch.empty(size(handle(), cache, new, Hq, 1), dtype=torch.uint8, device="cuda")
    start, length = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, new], [ctx]))
    out, lse = torch.empty_like(q), torch.empty((new, Hq), device="cuda")
    width = table.numel()
    before = b.awe_launch_count(handle())
    attention(handle(), cache, q, b.BF16, new, Hq, Hq * D, start, length, 1, table, width, width, D ** -0.5, True, window, out, Hq * D, lse, ws)
    torch.cuda.synchronize()
    assert b.awe_last_device_status(handle()) == (0, 0)
    return out, lse, b.awe_launch_count(handle()) - before


@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("new,window", [(3, 300), (700, 1000), (1, 0)])
def test_contexts_that_end_16_tokens_below_2_to_the_31(new, window, four):
    """With a window as a short context that ends alike; the whole of it as one page that 2^27 - 1 table entries name: its logarithm is the page's and
    that of their number, but for the sum of so many FP32 terms."""
    n, D = 2 ** 27 - 1, 64
    g = torch.Generator(device="cuda").manual_seed(new)
    q = torch.empty((new, 8, D), device="cuda").normal_(generator=g).to(torch.bfloat16)
    if window:
        table = torch.arange(n, dtype=torch.int32, device="cuda").remainder_(40)
        out, lse, launches = long_call(four, D, 40, table, q, new, 16 * n, window)
        assert (launches == 3) == (new == 700)
        # the same steps: 2,160 tokens end as far behind a multiple of 128 as 2^31 - 16 do
        short = table[-135:].clone()
        want, want_lse, launches = long_call(four, D, 40, torch.cat([short, short.new_full((5000,), -1)]), q, new, 16 * 135, window)
        assert (launches == 3) == (new == 700)
        assert torch.equal(lse, want_lse) and torch.equal(out, want)
    else:
        table = torch.zeros(n, dtype=torch.int32, device="cuda")
        out, lse, _ = long_call(four, D, 40, table, q, new, 16 * n, 0)
        want, want_lse, _ = long_call(four, D, 40, table[:1], q, new, 16, 0)
        assert float((lse - want_lse - math.log(n)).abs().max()) < 0.02
        assert float((out.double() - want.double()).abs().max()) <= 0.02 * float(want.abs().max())


@pytest.mark.parametrize("exponent,scale", [(e, s) for e in (100, 120, 125, 126, -100, -120) for s in (1.0, 0.125, 2.0 ** -20)
                                            if 4 * 2.0 ** e * s < 2.0 ** 128])  # the score in the kernel's unit
@pytest.mark.parametrize("D", [64, 128, 256])
def test_queries_at_the_ends_of_the_range(D, exponent, scale):
    """BF16 queries of one element 2^exponent: one token's score is that times scale and the others' are 0, or all are 0 but for bits that count
    for nothing.  Finite, and the one token's values alone where its score is large."""
    s = built([0.0] * 9 + [8.0] + [0.0] * 30, [1.0] * 40, [1.0], D, b.BF16, wide=False)
    s["q"][:, :, 0] = 2.0 ** exponent
    s["scale"] = scale * math.log(2.0)
    out, lse, _ = attend(s)
    want, want_lse, size, _, _ = reference(s)
    assert bool(((out - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -14) * (1 + 2.0 ** -8) * size).all())
    assert bool(((lse - want_lse).abs() <= 2.0 ** -14 + 2.0 ** -21 * want_lse.abs()).all())


@pytest.mark.parametrize("n", [1, 40, 300])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_scores_next_to_the_lowest_number(D, n):
    """Every token's score is -3.75 2^126 = -3.19e38: they weigh alike."""
    s = built([7.6] * n, [1.0] * n, [1.0], D, b.BF16, wide=False)
    s["q"][:, :, 0] = -2.0 ** 126
    out, lse, _ = attend(s)
    want, want_lse, size, _, _ = reference(s)
    assert bool((want_lse / math.log(2.0) < -3.1e38).all())
    assert bool(((out - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -11 + 2.0 ** -14) * (1 + 2.0 ** -8) * size).all())
    assert bool(((lse - want_lse).abs() <= 2.0 ** -21 * want_lse.abs()).all())


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("new,ctx,D", [(1, 777, 64), (1, 3000, 128), (2, 900, 256), (600, 1500, 128), (1024, 1024, 64)])
@pytest.mark.parametrize("spread", [0.1, 1.0, 6.0])
def test_errors_as_a_root_mean_square(spread, new, ctx, D, dtype):
    """Weights are off by 2^-11 of themselves at most and independently of one another, so that an output's error has a root mean square below
    2^-11 sqrt(sum (p v)^2), and its rounding one below u |out|.  A score of S in base 2 is rounded by 2^-24 S, a few times over, which with the
    exponentials and the sums is less than 2^-16 of a weight up to S = 2^6 (ln 2 2^-18 a rounding) and in proportion above.  Two floors: weights below
    2^-23 of the largest, P, are off by 2^-34 P (as above; for few rows of the largest product with a value's scale, and scales differ by less than
    2^5 here), and FP16 outputs below its normal range by 2^-25."""
    s = make([new], [ctx], 8, 2, D, 16, dtype, seed=D + new, spread=spread, width=4096 // 16 if new > 2 else None)
    assert (call(s) == 3) == (new > 2)
    u = torch.finfo(TORCH[dtype]).eps / 2
    pages = s["table"][0, :-(-ctx // 16)].long()
    hidden = torch.arange(ctx, device="cuda") > torch.arange(ctx - new, ctx, device="cuda")[:, None]
    total = count = 0.0
    for h in range(2):
        k, v = (values(s[a][pages, h], s[a + "p"][pages, h]).reshape(-1, D)[:ctx] for a in "kv")
        for i in range(4 * h, 4 * h + 4):
            x = (s["q"][:, i * D:(i + 1) * D].double() @ k.t() * s["scale"]).masked_fill(hidden, -math.inf)
            p = torch.softmax(x, 1)
            want = p @ v
            most, high = p.amax(1, keepdim=True), max(1.0, float(x.masked_fill(hidden, 0.0).abs().max()) / math.log(2.0) / 2 ** 6)
            floor = 2.0 ** -34 * (2 ** 5 if new <= 2 else 1) * most * ((p < 2.0 ** -23 * most).double() @ v.square()).sqrt() + 2.0 ** -25
            size = 2.0 ** -11 * (p.square() @ v.square()).sqrt() + u * want.abs() + 2.0 ** -16 * high * (p @ v.abs()) + floor
            total += float(((s["out"][:new, i * D:(i + 1) * D].double() - want) / size).square().sum())
            count += want.numel()
            lse = torch.logsumexp(x, 1)
            assert float((s["lse"][:new, i].double() - lse).square().mean().sqrt()) <= 2.0 ** -18 * high + 2.0 ** -22 * float(lse.abs().max())
    assert math.sqrt(total / count) <= 1.0


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,H", [(1, 1), (8, 2), (16, 1)])
@pytest.mark.parametrize("new,ctx,window", [(1, 1, 0), (1, 2, 0), (1, 900, 1), (3, 3, 0), (1, 777, 0), (1, 5000, 0), (6, 300, 40)])
def test_fp16_outputs_of_few_rows_are_rounded_once(new, ctx, window, Hq, H, D):
    """A weight is off by 2^-22 of itself beside the output's own rounding, u |out|: scores below 2^5, exponentials and sums add less than 2^-17 of
    sum p |v|.  Of one token the output is its values."""
    s = make([new], [ctx], Hq, H, D, 16, b.F16, window, seed=D + ctx)
    call(s)
    u, G = 2.0 ** -11, Hq // H
    pages = s["table"][0, :-(-ctx // 16)].long()
    tok, pos = torch.arange(ctx, device="cuda"), torch.arange(ctx - new, ctx, device="cuda")[:, None]
    hidden = (tok > pos) | ((tok <= pos - window) if window else torch.zeros_like(tok > pos))
    for h in range(H):
        k, v = (values(s[a][pages, h], s[a + "p"][pages, h]).reshape(-1, D)[:ctx] for a in "kv")
        for i in range(G * h, G * h + G):
            x = (s["q"][:, i * D:(i + 1) * D].double() @ k.t() * s["scale"]).masked_fill(hidden, -math.inf)
            assert float(x.masked_fill(hidden, 0.0).abs().max()) < 2 ** 5 * math.log(2.0)
            p = torch.softmax(x, 1)
            want, got = p @ v, s["out"][:new, i * D:(i + 1) * D].double()
            assert bool(((got - want).abs() <= u * want.abs() + (1 + u) * 2.0 ** -17 * (p @ v.abs()) + 2.0 ** -25).all())
            if ctx == 1 or window == 1:
                assert torch.equal(got, v[-1:].half().double())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,ctx,window", [(1500, 1500, 0), (1500, 3000, 1), (2000, 2500, 3), (1500, 1600, 20)])
def test_fp16_prompts_rows_of_few_tokens(new, ctx, window, D):
    """Rows that see one token have its values; of few, the weights' roundings (2^-11 of each, d_j) are off by sum p_j d_j (v_j - out), and the output's
    own by u |out|: scores, exponentials and sums add less than 2^-17 of sum p |v|."""
    s = make([new], [ctx], 8, 2, D, 16, b.F16, window, seed=D + ctx, width=256)
    assert call(s) == 3
    u = 2.0 ** -11
    pages = s["table"][0, :-(-ctx // 16)].long()
    tok, pos = torch.arange(ctx, device="cuda"), torch.arange(ctx - new, ctx, device="cuda")[:, None]
    seen = (tok <= pos) & ((tok > pos - window) if window else torch.ones_like(tok <= pos))
    few = seen.sum(1) < 32
    assert bool(few.any())
    for h in range(2):
        k, v = (values(s[a][pages, h], s[a + "p"][pages, h]).reshape(-1, D)[:ctx] for a in "kv")
        for i in range(4 * h, 4 * h + 4):
            x = (s["q"][:, i * D:(i + 1) * D].double() @ k.t() * s["scale"]).masked_fill(~seen, -math.inf)[few]
            p = torch.softmax(x, 1)
            want, got = p @ v, s["out"][:new, i * D:(i + 1) * D].double()[few]
            for r0 in range(0, len(p), 256):
                q, w = p[r0:r0 + 256], want[r0:r0 + 256]
                near = q.sum(0) > 0
                spread = torch.einsum("rn,rnd->rd", q[:, near], (v[near] - w[:, None]).abs())
                bound = u * w.abs() + (1 + u) * (u * spread + 2.0 ** -17 * (q @ v.abs())) + 2.0 ** -25
                assert bool(((got[r0:r0 + 256] - w).abs() <= bound).all())
            one = seen[few].sum(1) == 1
            assert torch.equal(got[one], (seen[few][one].double() @ v).half().double())
