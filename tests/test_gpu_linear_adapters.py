"""awe_linear_adapters against y = base + scale * B (A x) in 64 bits.

Tolerance.  With u = A x: FP32 sums of K exact products, in some order, are off by at most K 2^-23 sum |a x| (each addition rounds or cuts
off at most an ulp); the two 16-bit values hold u to 2^-16 of the token's largest |scale u|; the second sum is off by at most
rank 2^-23 of its terms; y is rounded by eps / 2."""
import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle

pytestmark = pytest.mark.gpu
TORCH = {b.F16: torch.float16, b.BF16: torch.bfloat16, b.F32: torch.float32}


def make(lengths, which, rank, N, K, dtype, out, seed=0, pad=0, n_adapters=5, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.empty(s, device="cuda").normal_(generator=g)  # noqa: E731
    T, t = sum(lengths), TORCH[dtype]
    start = [0]
    for n in lengths:
        start.append(start[-1] + n)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(T=T, B=len(lengths), rank=rank, N=N, K=K, dtype=dtype, out=out, L=n_adapters, lengths=lengths, which=which,
                x=draw(T, K + pad).to(t), a=(draw(n_adapters, rank, K) * K ** -0.5).to(t), b=(draw(n_adapters, N, rank) * rank ** -0.5).to(t),
                scale=torch.rand(n_adapters, generator=g, device="cuda") + 0.5 if scale else None, base=draw(T, N).to(TORCH[out]),
                start=ints(start), adapter=ints(which), y=torch.full((T, N), 7.0, device="cuda").to(TORCH[out]))


def call(s, base="base", y=None, stream=None):
    L = b.adapters(s["a"], s["b"], s["scale"], s["dtype"], s["L"], s["rank"], s["N"], s["K"])
    y = s["y"] if y is None else y
    src = {"base": s["base"], "none": None, "y": y}[base]
    b.awe_linear_adapters(handle(), L, s["x"], s["T"], s["x"].stride(0), s["start"], s["adapter"], s["B"], src, s["N"], y, s["out"], y.stride(0), stream)
    return y


def check(s, y, base=None):
    at = 0
    base = s["base"] if base is None else base
    eps = torch.finfo(TORCH[s["out"]]).eps / 2
    for n, i in zip(s["lengths"], s["which"]):
        rows = slice(at, at + n)
        at += n
        want, slack = base[rows].double(), torch.zeros((), device="cuda", dtype=torch.float64)
        if 0 <= i < s["L"] and n:
            x, A, B = s["x"][rows, :s["K"]].double(), s["a"][i].double(), s["b"][i].double()
            f = float(s["scale"][i]) if s["scale"] is not None else 1.0
            u = f * (x @ A.t())
            u_off = f * s["K"] * 2.0 ** -23 * (x.abs() @ A.abs().t()) + 2.0 ** -16 * u.abs().amax(1, keepdim=True) + 2.0 ** -23 * u.abs()
            want = want + u @ B.t()
            slack = u_off @ B.abs().t() + (2 * s["rank"] + 2) * 2.0 ** -23 * (u.abs() @ B.abs().t()) + 2.0 ** -23 * base[rows].double().abs()
        assert bool(((y[rows].double() - want).abs() <= slack + eps * (want.abs() + slack)).all()), (i, n)


@pytest.mark.parametrize("dtype,out", [(b.BF16, b.BF16), (b.F16, b.F16), (b.BF16, b.F32), (b.F16, b.F32)])
@pytest.mark.parametrize("rank", [8, 16, 24, 40, 64, 72, 128])
def test_single_tokens(rank, dtype, out):
    s = make([1] * 7, [0, 3, -1, 3, 4, 5, 1], rank, 517, 264, dtype, out, seed=rank)
    check(s, call(s))


@pytest.mark.parametrize("rank", [8, 16, 32, 56, 128])
@pytest.mark.parametrize("dtype,out,N", [(b.BF16, b.BF16, 640), (b.F16, b.F16, 517), (b.BF16, b.F32, 256), (b.F16, b.F32, 333)])
def test_prompts(rank, dtype, out, N):
    s = make([33, 0, 1, 64, 100, 31, 8], [1, 2, 0, 4, -1, 3, 3], rank, N, 528, dtype, out, seed=rank + N, pad=8)
    check(s, call(s))


@pytest.mark.parametrize("lengths", [[1], [8], [9], [0, 0, 5], [32] * 40, [1] * 300, [2, 0, 16, 7, 1, 1, 8, 3] * 9, [200]])
def test_lengths_of_many_kinds(lengths):
    s = make(lengths, [(3 * i) % 6 - 1 for i in range(len(lengths))], 16, 136, 72, b.BF16, b.F32, seed=len(lengths))
    check(s, call(s))


def test_all_numbers_of_blocks_a_cluster():
    """From one block for each of many requests to sixteen for one."""
    for B in (1, 5, 20, 40, 100, 300):
        s = make([1] * B, [i % 5 for i in range(B)], 8, 300, 4096, b.F16, b.F32, seed=B)
        check(s, call(s))
        s = make([12] * B, [i % 5 for i in range(B)], 8, 300, 4096, b.BF16, b.BF16, seed=B)
        check(s, call(s))


def test_long_sums_and_wide_results():
    for T in (1, 40):
        s = make([T], [2], 64, 8200, 8200, b.F16, b.F16, seed=T)
        check(s, call(s))


@pytest.mark.parametrize("T", [3, 50])
def test_base_in_place_without_a_base_and_without_scales(T):
    s = make([T, 1], [1, -1], 16, 264, 64, b.BF16, b.BF16, seed=T, scale=False)
    check(s, call(s, "none"), torch.zeros_like(s["base"]))
    y = s["base"].clone()
    check(s, call(s, "y", y))


@pytest.mark.parametrize("lengths", [[2, 1], [40, 9]])
def test_rows_outside_the_requests_and_between_the_rows_stay(lengths):
    s = make(lengths, [0, 1], 16, 100, 64, b.F16, b.F16)
    wide = torch.full((s["T"], 108), 7.0, device="cuda", dtype=torch.float16)
    s["start"] = s["start"].clamp(max=s["T"] - 1)  # the last row belongs to nobody
    y = call(s, y=wide)
    s["lengths"] = [lengths[0], lengths[1] - 1]
    check(s, y[:, :100])
    assert bool((y[-1] == 7.0).all()) and bool((y[:, 100:] == 7.0).all())


def test_large_and_small_sums_of_fp16_adapters():
    for factor in (2.0 ** -12, 2.0 ** 6):  # u beyond 65,504 and near 2^-24
        s = make([5, 40], [0, 1], 32, 200, 512, b.F16, b.F32, seed=3)
        s["a"] = (s["a"].float() * 512 ** 0.5 * factor).to(torch.float16)
        s["x"] = (s["x"].float() * factor * 8).to(torch.float16)
        check(s, call(s))


def test_the_same_twice_and_from_a_graph_with_other_data():
    for lengths in ([1, 1, 3], [70, 33]):
        s = make(lengths, [0, 2, 1][:len(lengths)], 24, 300, 256, b.BF16, b.BF16)
        first = call(s).clone()
        assert torch.equal(first, call(s))
        stream = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call(s)
        s["x"].copy_(s["x"].flip(0))
        s["adapter"].fill_(3)
        s["which"] = [3] * len(lengths)
        graph.replay()
        torch.cuda.synchronize()
        check(s, s["y"])


def test_refusals():
    s = make([2, 3], [0, 1], 16, 64, 64, b.BF16, b.BF16)

    def refused(status, **changed):
        with pytest.raises(b.AweError) as e:
            t = {**s, **changed}
            L = b.adapters(t["a"], t["b"], t["scale"], t["dtype"], t["L"], t["rank"], t["N"], t["K"])
            b.awe_linear_adapters(handle(), L, t["x"], t["T"], t.get("ldx", t["K"]), t["start"], t["adapter"], t["B"], t["base"], t.get("ldb", t["N"]), t["y"],
                                  t["out"], t.get("ldy", t["N"]))
        assert e.value.status == status, changed

    invalid, unsupported, alignment = 1, 2, b_alignment()
    for changed in (dict(T=-1), dict(B=-1), dict(N=0), dict(K=0), dict(L=0), dict(rank=0), dict(x=None), dict(y=None), dict(start=None), dict(adapter=None),
                    dict(ldx=56), dict(ldy=63), dict(ldb=63), dict(dtype=3), dict(out=-1), dict(base=s["y"], ldb=72), dict(a=None), dict(b=None)):
        refused(invalid, **changed)
    for changed in (dict(rank=12), dict(rank=136), dict(K=60, ldx=64), dict(dtype=b.F32), dict(out=b.F16), dict(B=b.KV_MAX_REQUESTS + 1)):
        refused(unsupported, **changed)
    for changed in (dict(x=s["x"].view(-1)[1:]), dict(ldx=68), dict(a=s["a"].view(-1)[1:])):
        refused(alignment, **changed)
    empty = dict(s, T=0)
    call(empty)
    empty = dict(s, B=0)
    before = s["y"].clone()
    call(empty)
    assert torch.equal(before, s["y"])


def b_alignment():
    return next(i for i in range(1, 12) if "align" in b.status_string(i))


@pytest.mark.parametrize("rank", [8, 16, 32, 56, 128])
@pytest.mark.parametrize("dtype,out,N", [(b.BF16, b.BF16, 640), (b.F16, b.F16, 517), (b.BF16, b.F32, 256), (b.F16, b.F32, 333)])
def test_long_prompts(rank, dtype, out, N):
    """As many tokens as take units of 32, of every length of the last one."""
    s = make([33, 0, 1, 64, 300, 31, 8, 500, 207], [1, 2, 0, 4, -1, 3, 3, 0, 2], rank, N, 528, dtype, out, seed=rank + N, pad=8)
    y = call(s).clone()
    check(s, y)
    assert torch.equal(y, call(s))


@pytest.mark.parametrize("lengths", [[32] * 40, list(range(1, 65)), [2000], [0] * 9 + [641, 0, 700]])
def test_long_prompts_of_many_lengths(lengths):
    s = make(lengths, [(3 * i) % 6 - 1 if len(lengths) > 1 else 2 for i in range(len(lengths))], 16, 136, 4104, b.BF16, b.F32, seed=len(lengths))
    check(s, call(s))
    check(s, call(s, "none"), torch.zeros_like(s["base"]))
    y = s["base"].clone()
    check(s, call(s, "y", y))


def test_long_prompts_outside_the_requests_and_between_the_rows():
    s = make([400, 500], [0, 1], 16, 100, 64, b.F16, b.F16)
    wide = torch.full((s["T"], 108), 7.0, device="cuda", dtype=torch.float16)
    s["start"] = s["start"].clamp(max=s["T"] - 1)
    y = call(s, y=wide)
    s["lengths"] = [400, 499]
    check(s, y[:, :100])
    assert bool((y[-1] == 7.0).all()) and bool((y[:, 100:] == 7.0).all())


def test_large_and_small_sums_of_long_prompts():
    for factor in (2.0 ** -12, 2.0 ** 6):
        s = make([5, 640], [0, 1], 32, 200, 512, b.F16, b.F32, seed=3)
        s["a"] = (s["a"].float() * 512 ** 0.5 * factor).to(torch.float16)
        s["x"] = (s["x"].float() * factor * 8).to(torch.float16)
        check(s, call(s))


@pytest.mark.parametrize("dtype", [b.BF16, b.F16])
@pytest.mark.parametrize("lengths", [[3, 1, 4], [300, 1, 407]])
def test_infinities_and_nan_stay_with_their_token(lengths, dtype):
    s = make(lengths, [0, -1, 1], 24, 200, 512, dtype, dtype, seed=7)
    s["x"][1, 40], s["x"][-1, 511], s["x"][lengths[0], 3] = float("inf"), float("nan"), float("nan")  # the last of a token without an adapter
    y = call(s).clone()
    bad = torch.zeros(s["T"], dtype=torch.bool, device="cuda")
    bad[1] = bad[-1] = True
    assert not bool(y[bad].isfinite().any()) and bool(y[~bad].isfinite().all())
    s["x"][bad] = 0
    s["x"][lengths[0], 3] = 0
    assert torch.equal(call(s)[~bad], y[~bad])
