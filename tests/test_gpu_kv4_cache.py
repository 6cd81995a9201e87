"""awe_kv4_append and awe_kv4_read: exactly the values of the definition (each FP32 step of it rounded alike here), which are
within half a scale of the rotated rows in 64 bits.

Tolerance of that: the rotation's two products and their sum round by 2^-24 of |a cos| + |b sin| each, the quotients next to a tie by an ulp."""
import math

import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle

pytestmark = pytest.mark.gpu
TORCH = {b.F16: torch.float16, b.BF16: torch.bfloat16}


def angles(count, dim):
    step = 10000.0 ** (-torch.arange(0, dim, 2, dtype=torch.float64, device="cuda") / dim)
    a = torch.arange(count, dtype=torch.float64, device="cuda")[:, None] * step
    return torch.cat([a.cos(), a.sin()], 1).float()


def make(T, Hq, H, D, page, dtype, rotary, interleaved=False, seed=0, n_pages=None, n_positions=4000, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_pages = n_pages or -(-T // page) + 3
    slots = torch.randperm(n_pages * page, generator=g, device="cuda")[:T]
    rows = torch.empty((T, (Hq + 2 * H) * D + pad), device="cuda").normal_(generator=g)
    rows *= torch.empty((1, rows.shape[1]), device="cuda").normal_(generator=g).mul_(0.7).exp_()
    u8 = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda", dtype=torch.uint8)  # noqa: E731
    i16 = lambda *s: torch.randint(0, 20000, s, generator=g, device="cuda", dtype=torch.int16)  # noqa: E731
    return dict(T=T, Hq=Hq, H=H, D=D, page=page, dtype=dtype, rows=rows.to(TORCH[dtype]), slots=slots, n_pages=n_pages,
                k=u8(n_pages, H, page, D // 2), v=u8(n_pages, H, page, D // 2), kp=i16(n_pages, H, page), vp=i16(n_pages, H, page),
                positions=torch.randint(0, n_positions, (T,), generator=g, device="cuda", dtype=torch.int32), n_positions=n_positions,
                rotary=rotary, interleaved=interleaved, table=angles(n_positions, rotary) if rotary else None,
                q=torch.full((T, Hq * D), 7.0, device="cuda", dtype=TORCH[dtype]))


def cache_of(s):
    return b.kv4_cache(s["k"], s["v"], s["kp"], s["vp"], s["n_pages"], s["H"], s["page"], s["D"])


def append(s, stream=None):
    Hq, H, D, rows = s["Hq"], s["H"], s["D"], s["rows"]
    turn = b.rotary(s["table"], s["n_positions"], s["rotary"], s["interleaved"]) if s["rotary"] else None
    ld = rows.stride(0)
    b.awe_kv4_append(handle(), cache_of(s), turn, s["dtype"], s["T"], Hq, rows if Hq else None, ld, rows[:, Hq * D:], ld, rows[:, (Hq + H) * D:], ld,
                     s["positions"] if turn else None, s["slots"], s["q"] if Hq else None, Hq * D, stream)


def read(s, dtype=b.F16, slots=None):
    slots = s["slots"] if slots is None else slots
    k, v = (torch.full((slots.numel(), s["H"], s["D"]), 9.0, device="cuda", dtype=TORCH[dtype]) for _ in range(2))
    b.awe_kv4_read(handle(), cache_of(s), slots.numel(), slots, dtype, k, s["H"] * s["D"], v, s["H"] * s["D"])
    return k, v


def turned(s, dtype):
    """Queries and keys (T x heads x D) rotated in the given type, step by step."""
    H, Hq, D, half = s["H"], s["Hq"], s["D"], s["rotary"] // 2
    x = s["rows"][:, :(Hq + 2 * H) * D].to(dtype).view(s["T"], Hq + 2 * H, D).clone()
    if half:
        at = s["table"][s["positions"].long()].to(dtype)[:, None]
        cos, sin = at[..., :half], at[..., half:]
        i = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["interleaved"] else (slice(0, half), slice(half, 2 * half))
        p, q = x[:, :Hq + H, i[0]].clone(), x[:, :Hq + H, i[1]].clone()
        x[:, :Hq + H, i[0]], x[:, :Hq + H, i[1]] = p * cos - q * sin, q * cos + p * sin
    return x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]


def quantised(x):
    """Values, scales of rows in FP32, by the definition; NaN and infinities as it says."""
    finite = torch.where(x.isfinite(), x, 0.0)
    lo, hi = finite.amin(-1, keepdim=True).clamp(-30480.0, 0.0), finite.amax(-1, keepdim=True).clamp(0.0, 30480.0)
    raw = ((hi - lo) / torch.full_like(lo, 15.0)).clamp(min=2.0 ** -18)
    m, e = torch.frexp(raw)
    scale = torch.ldexp(torch.ceil(m * 128.0), e - 7)
    below = (lo / scale).round()
    return ((torch.nan_to_num(x, 0.0, math.inf, -math.inf) / scale).round() - below).clamp(0.0, 15.0).add(below) * scale, scale


def check(s, live=None):
    live = torch.ones(s["T"], dtype=torch.bool, device="cuda") if live is None else live
    q, k, v = turned(s, torch.float32)
    got_k, got_v = read(s)
    for got, x in ((got_k, k), (got_v, v)):
        value, scale = quantised(x)
        assert torch.equal(got[live].float(), value[live]), (got[live].float() - value[live]).abs().max()
        assert torch.equal(value.half().float(), value)  # FP16 holds them
    if s["Hq"]:
        assert torch.equal(s["q"].view(s["T"], s["Hq"], -1)[live], q.to(TORCH[s["dtype"]])[live])
    exact_q, exact_k, exact_v = turned(s, torch.float64)
    for got, x in ((got_k, exact_k), (got_v, exact_v)):
        _, scale = quantised(x.float())
        inside = live & (x.abs().amax((1, 2)) < 30000)
        largest = x.abs().amax(-1, keepdim=True)
        assert bool(((got.double() - x).abs() <= scale / 2 * (1 + 2.0 ** -20) + 2.0 ** -21 * largest)[inside].all())


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
@pytest.mark.parametrize("T,Hq,H,D,page,rotary,interleaved", [
    (1, 4, 1, 64, 16, 64, False), (1, 32, 8, 128, 16, 128, True), (7, 5, 1, 256, 32, 256, False), (33, 8, 2, 128, 64, 64, True),
    (19, 3, 3, 64, 256, 24, False), (5, 9, 3, 128, 16, 8, False), (6, 0, 2, 64, 16, 0, False), (64, 32, 8, 128, 16, 128, False),
    (1500, 16, 4, 128, 128, 96, True), (700, 10, 2, 256, 32, 48, False), (900, 2, 1, 64, 16, 0, False), (3, 128, 128, 256, 16, 256, True)])
def test_append_and_read(T, Hq, H, D, page, rotary, interleaved, dtype):
    s = make(T, Hq, H, D, page, dtype, rotary, interleaved, seed=T, pad=8 * (T % 3))
    append(s)
    check(s)


@pytest.mark.parametrize("D,H,rotary,interleaved", [(64, 3, 64, False), (128, 2, 32, True), (256, 1, 256, False)])
def test_many_tokens_with_some_left_out(D, H, rotary, interleaved):
    """So many that a block takes several tokens; their number is no multiple of that, and any of a block's may be left out."""
    T = 2603
    s = make(T, 5, H, D, 32, b.BF16, rotary, interleaved, seed=D)
    g = torch.Generator(device="cuda").manual_seed(1)
    out = torch.rand(T, generator=g, device="cuda")
    slots, positions = s["slots"].clone(), s["positions"].clone()
    s["slots"][out < 0.2] = -1
    s["positions"][(out > 0.1) & (out < 0.3)] = -1
    append(s)
    turned_rows = (out <= 0.1) | (out >= 0.3)
    stored = turned_rows & (out >= 0.2)
    q = s["q"].clone()
    s["positions"], s["slots"] = positions, slots
    want = turned(s, torch.float32)[0].to(torch.bfloat16).view(T, -1)
    assert torch.equal(q[turned_rows], want[turned_rows]) and bool((q[~turned_rows] == 7.0).all())
    s["q"] = want
    check(s, stored)


def test_far_positions():
    s = make(40, 2, 1, 128, 16, b.BF16, 128, n_positions=300000)
    s["positions"] += 299990 - s["positions"].max()
    append(s)
    check(s)


@pytest.mark.parametrize("dtype", [b.F16, b.BF16])
def test_rows_of_all_kinds(dtype):
    """Constant, one-sided, tiny, huge, empty and special rows, and values that lie on ties."""
    s = make(16, 1, 1, 64, 16, dtype, 0)
    x = s["rows"]
    v = x[:, 128:]
    v[0] = 0.0
    v[1] = 3.0
    v[2] = -0.37
    v[3] = v[3].abs()
    v[4] = -v[4].abs()
    v[5] *= 2.0 ** -14
    v[6] *= 2.0 ** -26 if dtype == b.F16 else 2.0 ** -60
    v[7] = torch.where(torch.arange(64, device="cuda") % 2 == 0, 60000.0, -60000.0)
    v[8, ::2], v[8, 1::2] = 65000.0 if dtype == b.F16 else 1e30, 1.0
    v[9] = torch.arange(64, device="cuda") * 0.5 - 7.5  # scale 2.1: multiples of a half
    v[10] = torch.arange(64, device="cuda") % 31 * 0.5  # scale 1: every other value is a tie
    v[11] = -(torch.arange(64, device="cuda") % 31 * 0.5)
    v[12, 3] = math.nan
    v[13, 5], v[13, 6] = math.inf, -math.inf
    v[14] = math.nan
    v[15] = -math.inf
    append(s)
    check(s)
    k, got = read(s)
    at = {int(t): i for i, t in enumerate(range(16))}
    assert float(got[at[12], 0, 3]) == 0.0 and not bool(got[at[14]].any())
    assert float(got[at[13], 0, 5]) == float(got[at[13], 0].max()) and float(got[at[13], 0, 6]) == float(got[at[13], 0].min())


def test_tokens_left_out():
    """Skipped slots, slots outside the pool and positions outside the table; nothing else of the pool changes."""
    s = make(12, 2, 2, 64, 16, b.F16, 64)
    before = {n: s[n].clone() for n in ("k", "v", "kp", "vp")}
    slots, positions = s["slots"].clone(), s["positions"].clone()
    s["slots"][1], s["slots"][2] = -1, s["n_pages"] * 16
    s["positions"][4], s["positions"][5] = -1, s["n_positions"]
    append(s)
    stored = torch.ones(12, dtype=torch.bool, device="cuda")
    stored[[1, 2, 4, 5]] = False
    q = s["q"].clone()
    assert bool((q[4] == 7.0).all()) and bool((q[5] == 7.0).all())
    queries = stored.clone()
    queries[[1, 2]] = True
    want, _, _ = turned({**s, "positions": s["positions"].clamp(0, s["n_positions"] - 1)}, torch.float32)
    assert torch.equal(q.view(12, 2, 64)[queries], want.half()[queries])
    s["positions"] = positions
    k, v = read(s)
    assert bool((k[1] == 9.0).all()) and bool((v[2] == 9.0).all())
    s["slots"] = slots
    check({**s, "Hq": 2, "q": want.half().view(12, -1)}, stored)
    touched = torch.zeros(s["n_pages"] * 16, dtype=torch.bool, device="cuda")
    touched[slots[stored]] = True
    for n in before:
        same = (s[n] == before[n]).view(s["n_pages"], 2, 16, -1).all(-1)
        assert bool((same | touched.view(-1, 1, 16)).all()), n


def test_queries_in_place_keys_alone_and_bf16_read():
    s = make(50, 4, 2, 128, 16, b.BF16, 128)
    keep = s["rows"].clone()
    turn = b.rotary(s["table"], s["n_positions"], 128, False)
    ld = s["rows"].stride(0)
    b.awe_kv4_append(handle(), cache_of(s), turn, b.BF16, 50, 4, s["rows"], ld, s["rows"][:, 512:], ld, s["rows"][:, 768:], ld, s["positions"], s["slots"],
                     s["rows"], ld)
    s["q"] = s["rows"][:, :512].clone()
    assert torch.equal(s["rows"][:, 512:], keep[:, 512:])
    s["rows"] = keep
    check(s)
    k, _ = read(s)
    k2, _ = read(s, b.BF16)
    assert torch.equal(k2, k.bfloat16())
    only = torch.zeros_like(k)
    b.awe_kv4_read(handle(), cache_of(s), 50, s["slots"], b.F16, None, 0, only, 256)
    assert torch.equal(only, read(s)[1])


def test_from_a_graph_on_another_stream():
    s = make(30, 4, 2, 64, 16, b.F16, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        append(s)
    s["rows"].copy_(s["rows"].flip(0))
    s["slots"].copy_(s["slots"].roll(1))
    graph.replay()
    torch.cuda.synchronize()
    check(s)


def test_refusals():
    s = make(4, 2, 1, 64, 16, b.F16, 64)
    wide = s["rows"].stride(0)

    def status(cache=None, turn=None, dtype=b.F16, T=4, Hq=2, q=s["rows"], ldq=wide, k=s["rows"], ldk=wide, positions=s["positions"], slots=s["slots"],
               out=s["q"], ldqo=128, **of_cache):
        c = {**dict(k=s["k"], v=s["v"], kp=s["kp"], vp=s["vp"], n_pages=s["n_pages"], H=1, page=16, D=64), **of_cache}
        cache = b.kv4_cache(c["k"], c["v"], c["kp"], c["vp"], c["n_pages"], c["H"], c["page"], c["D"])
        turn = turn or b.rotary(s["table"], s["n_positions"], 64)
        try:
            b.awe_kv4_append(handle(), cache, turn, dtype, T, Hq, q, ldq, k, ldk, s["rows"], wide, positions, slots, out, ldqo)
        except b.AweError as e:
            return e.status
        return b.OK

    assert status() == b.OK and status(T=0) == b.OK
    for bad in (dict(T=-1), dict(Hq=-1), dict(dtype=5), dict(k=None), dict(slots=None), dict(positions=None), dict(q=None), dict(out=None), dict(ldk=56),
                dict(ldq=120), dict(ldqo=120), dict(out=s["rows"], ldqo=128), dict(n_pages=0), dict(H=0), dict(kp=None),
                dict(turn=b.rotary(None, 10, 64)), dict(turn=b.rotary(s["table"], 0, 64)), dict(turn=b.rotary(s["table"], 10, 72))):
        assert status(**bad) == 1, bad
    for bad in (dict(dtype=b.F32), dict(page=8), dict(page=48), dict(page=512), dict(D=96), dict(turn=b.rotary(s["table"], 10, 12))):
        assert status(**bad) == 2, bad
    flat = s["rows"].view(-1)
    for bad in (dict(q=flat[4:]), dict(ldq=260), dict(k=flat[1:]), dict(ldk=260), dict(out=flat[2:]), dict(turn=b.rotary(s["table"].view(-1)[1:], 10, 64)),
                dict(kp=s["kp"].view(-1)[1:])):
        assert status(**bad) == 4, bad
    with pytest.raises(b.AweError):
        b.awe_kv4_read(handle(), cache_of(s), 4, None, b.F16, s["q"], 64, None, 0)
    with pytest.raises(b.AweError):
        b.awe_kv4_read(handle(), cache_of(s), 4, s["slots"], b.F32, s["q"], 64, None, 0)
    with pytest.raises(b.AweError):
        b.awe_kv4_read(handle(), cache_of(s), 4, s["slots"], b.F16, s["q"], 68, None, 0)
    b.awe_kv4_read(handle(), cache_of(s), 4, s["slots"], b.F16, None, 0, None, 0)
