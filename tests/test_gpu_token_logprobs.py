"""awe_token_logprobs against log-softmax in 64 bits.

Tolerance.  With d_j = scale (x_j - M) <= 0 and z = ln sum e^d: a term 2^t is off by 2^-22 + |t| 2^-23 of itself (exponential, FMA, the rounded
factor), the sums of n terms by n / 256 additions of a thread, at most 64 more, 2^-24 each; z by that and its own rounding.  Log probabilities
and lse are z plus one FMA.  That is below (2^-21 + (n / 256 + 64) 2^-24) (1 + |t|) for the terms that count (|t| < 32 here)."""
import math

import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle

pytestmark = pytest.mark.gpu
TORCH = {b.F16: torch.float16, b.BF16: torch.bfloat16, b.F32: torch.float32}


def logits(T, V, dtype, seed=0, pad=0, spread=2.0, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.empty(T * (V + pad) + offset, device="cuda").normal_(0.0, spread, generator=g).to(TORCH[dtype])
    return flat[offset:].view(T, V + pad)


def call(x, V, dtype, top, scale=1.0, tokens=None, stream=None):
    T = x.shape[0]
    f = lambda *s: torch.full(s, 99.0, device="cuda")  # noqa: E731
    out = dict(logprob=f(T), entropy=f(T), lse=f(T), top_logprob=f(T, top), top_id=torch.full((T, top), -5, dtype=torch.int32, device="cuda"))
    if tokens is None:
        tokens = torch.arange(T, device="cuda", dtype=torch.int32) * 7919 % V
    b.awe_token_logprobs(handle(), x, dtype, T, V, x.stride(0), scale, tokens, out["logprob"], out["entropy"], out["lse"], top, out["top_logprob"],
                         out["top_id"], stream)
    out["tokens"] = tokens
    return out


def check(out, x, V, scale=1.0):
    x = x[:, :V].double()
    T, top = out["top_id"].shape
    logp = torch.log_softmax(x * scale, 1)
    tol = (2.0 ** -21 + (V / 256 + 64) * 2.0 ** -24) * 33
    near = lambda got, want: bool(((got.double() - want).abs() <= tol + 2.0 ** -22 * want.abs()).all() or torch.equal(got.double(), want))  # noqa: E731
    token = out["tokens"].long()
    fine = (token >= 0) & (token < V)
    want = torch.where(fine, logp.gather(1, token.clamp(0, V - 1)[:, None])[:, 0], 0.0)
    masked = want == -math.inf
    assert torch.equal(out["logprob"].double() == -math.inf, masked) and near(out["logprob"][~masked], want[~masked])
    assert near(out["lse"], torch.logsumexp(x * scale, 1))
    entropy = -torch.where(logp > -math.inf, logp.exp() * logp, 0.0).sum(1)
    # each term's own error weighs p |t|: with the terms' as above, of the entropy itself
    assert near(out["entropy"], entropy)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    assert torch.equal(out["top_id"].long(), order)
    want = logp.gather(1, order)
    masked = want == -math.inf
    assert torch.equal(out["top_logprob"].double() == -math.inf, masked) and near(out["top_logprob"][~masked], want[~masked])


@pytest.mark.parametrize("dtype", [b.F16, b.BF16, b.F32])
@pytest.mark.parametrize("T,V", [(1, 1), (1, 7), (3, 33), (2, 1000), (5, 32003), (1, 131072), (70, 50257), (700, 2049)])
def test_sizes(T, V, dtype):
    x = logits(T, V, dtype, seed=V)
    top = min(20, V)
    check(call(x, V, dtype, top, 0.7), x, V, float(torch.tensor(0.7)))


@pytest.mark.parametrize("top", [0, 1, 2, 31, 32])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (7, 1)])
def test_alignments_and_numbers_of_alternatives(top, offset, pad):
    for dtype in (b.BF16, b.F32):
        x = logits(9, 4099, dtype, seed=top, pad=pad, offset=offset)
        check(call(x, 4099, dtype, top), x, 4099)


@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_equal_logits_in_any_order(V):
    """Ties go to the lower token, also -0 and 0, and where logits rise all along the row."""
    for dtype in (b.F16, b.F32):
        t = TORCH[dtype]
        rows = torch.stack([torch.zeros(V), torch.where(torch.arange(V) % 2 == 0, -0.0, 0.0), torch.arange(V) // 7 * 1.0 / V * 8, -(torch.arange(V) // 5) * 8.0 / V,
                            torch.where(torch.arange(V) == V - 1, 3.0, 1.0)]).to(t).cuda()
        check(call(rows, V, dtype, 32), rows, V)


def test_masked_tokens():
    """-inf has probability 0; a row with one token left, and one with none."""
    x = logits(6, 9000, b.BF16, seed=1)
    x[0] = -math.inf
    x[1] = -math.inf
    x[1, 8999] = 3.0
    x[2, ::2] = -math.inf
    x[3, 100:] = -math.inf
    x[4, :8990] = torch.finfo(torch.bfloat16).min
    tokens = torch.tensor([5, 8999, 4, 99, 8995, 9], dtype=torch.int32, device="cuda")
    out = call(x, 9000, b.BF16, 12, 1.0, tokens)
    check({k: v[1:] for k, v in out.items()}, x[1:], 9000)
    assert float(out["lse"][0]) == -math.inf and float(out["logprob"][0]) == -math.inf and float(out["entropy"][0]) == 0.0
    assert out["top_id"][0].tolist() == list(range(12)) and bool((out["top_logprob"][0] == -math.inf).all())


@pytest.mark.parametrize("where", [0, 3, 4500, 8999])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_with_nan_or_infinity(where, bad):
    x = logits(3, 9000, b.F16, seed=2)
    x[1, where] = bad
    out = call(x, 9000, b.F16, 5, 1.0, torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"))
    for k in ("logprob", "entropy", "lse", "top_logprob"):
        assert bool(out[k][1].isnan().all()), k
    rest = torch.where(x[1].isnan(), -math.inf, x[1]).double()
    assert out["top_id"][1].tolist() == torch.sort(rest, descending=True, stable=True).indices[:5].tolist()
    check({k: v[::2] for k, v in out.items()}, x[::2], 9000)
    x[1] = math.nan
    x[1, 6] = 1.0
    assert call(x, 9000, b.F16, 3)["top_id"][1].tolist() == [6, -1, -1]


def test_tokens_outside_and_outputs_not_wanted():
    x = logits(4, 600, b.F32)
    tokens = torch.tensor([-1, 600, 2 ** 31 - 1, 599], dtype=torch.int32, device="cuda")
    out = call(x, 600, b.F32, 3, 2.0, tokens)
    check(out, x, 600, 2.0)
    lse = torch.empty(4, device="cuda")
    b.awe_token_logprobs(handle(), x, b.F32, 4, 600, 600, 2.0, None, None, None, lse, 0, None, None)
    assert torch.equal(lse, out["lse"])
    ids = torch.empty((4, 3), dtype=torch.int32, device="cuda")
    b.awe_token_logprobs(handle(), x, b.F32, 4, 600, 600, 2.0, None, None, None, None, 3, None, ids)
    assert torch.equal(ids, out["top_id"])


def test_temperatures_and_large_logits():
    for scale in (0.01, 100.0):
        x = logits(3, 5000, b.F32, seed=5)
        x += 1000.0
        out = call(x, 5000, b.F32, 4, scale)
        want = torch.log_softmax(x.double() * float(torch.tensor(scale)), 1)
        got = out["top_logprob"].double()
        ref = want.gather(1, out["top_id"].long())
        # the logits' differences are exact in FP32; a term's exponent t is off by |t| 2^-22
        assert bool(((got - ref).abs() <= (2.0 ** -21 + 84 * 2.0 ** -24) * (1 + ref.abs()) * 33).all())


def test_the_same_twice_and_from_a_graph():
    for T in (1, 40):
        x = logits(T, 40000, b.BF16, seed=T)
        first, again = call(x, 40000, b.BF16, 20), call(x, 40000, b.BF16, 20)
        assert all(torch.equal(first[k], again[k]) for k in first)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            out = call(x, 40000, b.BF16, 20)
        x.copy_(x.flip(1))
        graph.replay()
        torch.cuda.synchronize()
        check(out, x, 40000)


def test_refusals():
    x = logits(2, 64, b.F32)
    f, i = torch.empty(2, 32, device="cuda"), torch.zeros(2, 32, dtype=torch.int32, device="cuda")

    def status(logits=x, dtype=b.F32, T=2, V=64, ld=64, scale=1.0, tokens=i, logprob=f, top=4):
        try:
            b.awe_token_logprobs(handle(), logits, dtype, T, V, ld, scale, tokens, logprob, None, None, top, f, i)
        except b.AweError as e:
            return e.status
        return b.OK

    assert status() == b.OK and status(T=0) == b.OK
    for bad in (dict(T=-1), dict(V=0), dict(ld=63), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(logits=None),
                dict(tokens=None), dict(top=-1), dict(V=3, top=4), dict(dtype=7)):
        assert status(**bad) == 1, bad
    assert status(top=33) == 2 and status(V=2 ** 30, ld=2 ** 30, T=1) == 2
    aligned = next(k for k in range(1, 12) if "align" in b.status_string(k))
    assert status(logits=x.view(torch.uint8).view(-1)[2:]) == aligned


@pytest.mark.parametrize("dtype", [b.F16, b.F32])
@pytest.mark.parametrize("T,V,top", [(1, 131072, 0), (3, 50257, 0), (2, 262147, 20), (70, 131075, 32), (100, 65601, 3), (160, 262144, 1), (301, 131072, 2)])
def test_long_rows_of_few_and_many_tokens(T, V, top, dtype):
    """Rows of one to eight blocks."""
    x = logits(T, V, dtype, seed=T)
    check(call(x, V, dtype, top, 0.7), x, V, float(torch.tensor(0.7)))


def test_two_streams_at_once():
    rows = [logits(33, 50257, b.BF16, seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in rows]
    torch.cuda.synchronize()
    out = [[], []]
    for _ in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                out[i].append(call(rows[i], 50257, b.BF16, 7))
    torch.cuda.synchronize()
    for i in range(2):
        check(out[i][0], rows[i], 50257)
        assert all(torch.equal(o[k], out[i][0][k]) for o in out[i] for k in o)
