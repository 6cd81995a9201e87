"""Log probabilities where they can go wrong: rows of which few tokens are left, masked by -inf or a type's lowest value, in either order of the work.
Alternatives are compared exactly, log probabilities as in test_gpu_token_logprobs."""
import math

import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .test_gpu_token_logprobs import TORCH, call, check, logits

pytestmark = pytest.mark.gpu


def top_of(x, V, top):
    """The stable order of a row's numbers; -1 where there are no more."""
    rows = []
    for row in x[:, :V].double():
        order = torch.sort(torch.where(row.isnan(), -math.inf, row), descending=True, stable=True).indices
        order = order[~row[order].isnan()][:top]
        rows.append(torch.cat([order, order.new_full((top - len(order),), -1)]))
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", [b.F16, b.BF16, b.F32])
@pytest.mark.parametrize("T,V", [(1, 131072), (70, 50257), (300, 3001), (2, 300), (3, 40)])
@pytest.mark.parametrize("live", [1, 5, 19, 20, 60, 400])
def test_few_tokens_left(live, T, V, dtype):
    """The others masked, by -inf or the type's lowest value; tokens left at the ends of the row, or with few threads."""
    top = min(20, V)
    full = logits(T, V, dtype, seed=live)
    g = torch.Generator(device="cuda").manual_seed(V)
    for lowest in (-math.inf, float(torch.finfo(TORCH[dtype]).min)):
        for kind in ("any", "front", "back", "stride"):
            if kind == "any":
                at = torch.rand((T, V), generator=g, device="cuda").topk(min(live, V), 1).indices
            else:
                at = {"front": torch.arange(live), "back": V - 1 - torch.arange(live), "stride": torch.arange(live) * 2048 % V}[kind].clamp(0, V - 1).cuda().expand(T, live)
            x = torch.full_like(full, lowest).scatter_(1, at, full.gather(1, at))
            out = call(x, V, dtype, top, 1.0, at[:, 0].to(torch.int32))
            check(out, x, V)


@pytest.mark.parametrize("top", [1, 2, 32])
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 0), (3, 5), (7, 1)])
def test_ends_of_rows_on_no_boundary(top, offset, pad):
    for dtype in (b.F16, b.F32):
        for V in (4099, 50):
            x = logits(9, V, dtype, seed=top, pad=pad, offset=offset)
            x[:, 3:V - 2] = -math.inf
            x[1::3, :] = 2.0
            x[2::3, :V // 2] = 5.0
            out = call(x, V, dtype, top)
            check(out, x, V)


@pytest.mark.parametrize("V", [9000, 50257])
@pytest.mark.parametrize("top", [1, 3, 32])
def test_nan_beside_equal_masked_and_other_tokens(top, V):
    for dtype in (b.BF16, b.F32):
        x = logits(8, V, dtype, seed=top)
        x[0, 17] = math.nan
        x[1] = -math.inf
        x[1, [5, 8000]] = torch.tensor([math.nan, 1.0], device="cuda").to(x.dtype)
        x[2] = 1.0
        x[2, ::3] = math.nan
        x[3, 2:] = math.nan
        x[4] = math.nan
        x[5, :] = math.inf
        x[6] = -math.inf
        x[6, 100] = math.inf
        x[7] = math.nan
        x[7, V - 1] = -math.inf
        out = call(x, V, dtype, top, 1.0, torch.zeros(8, dtype=torch.int32, device="cuda"))
        assert torch.equal(out["top_id"].long(), top_of(x, V, top))
        for k in ("logprob", "entropy", "lse"):
            assert bool(out[k].isnan().all()), k
        assert bool(out["top_logprob"].isnan().all())


@pytest.mark.parametrize("dtype", [b.F16, b.F32])
@pytest.mark.parametrize("top", [5, 20, 32])
def test_many_of_the_largest_with_few_threads(top, dtype):
    """A thread of a block takes 16 bytes of every 4,096: elements that large lie with `top` / 2 of 256 threads, more than there is room for."""
    V, each = 131072, 4 if dtype == b.F32 else 8
    x = logits(3, V, dtype, seed=top).clamp_(-20.0, 5.0)
    piece = torch.arange(V, device="cuda") // each % 256
    x[0] += torch.where(piece < max(2, top // 2), 30.0, 0.0).to(x.dtype)
    x[1] = torch.where(piece == 77, 40.0, x[1])
    x[2] = torch.where(piece < 2, torch.arange(V, device="cuda") % 97 / 8.0 + 20.0, x[2].float()).to(x.dtype)
    check(call(x, V, dtype, top), x, V)


def test_same_bits_again():
    x = logits(64, 50257, b.BF16, seed=3)
    x[::2, 40:] = -math.inf
    first, again = (call(x, 50257, b.BF16, 20) for _ in range(2))
    for k in first:
        assert torch.equal(first[k], again[k]), k


@pytest.mark.parametrize("dtype", [b.BF16, b.F32])
@pytest.mark.parametrize("T,V", [(64, 131072), (400, 32003)])
@pytest.mark.parametrize("spread", [0.1, 2.0])
def test_errors_of_many_tokens_as_a_root_mean_square(spread, T, V, dtype):
    """Of lse: its own rounding (below 16) 2^-21, the logarithm's 2^-20 (z below 12), the factor's, 2^-24 of t, whose mean is below log2 V ln 2 < 12,
    2^-20.4, the exponentials' bias 2^-22, and the sums': 512 additions of a thread are off by sqrt(512) 2^-24 of it as a root mean square, 256
    threads' together by 2^-23.5.  In all 2.6 2^-20.  Log probabilities (below 32) round by 2^-20 more; the entropy takes the factor's and the
    exponentials' errors times t once more, and its quotient's (below 17, times ln 2) 2^-21: below 4 2^-20."""
    x = logits(T, V, dtype, seed=V, spread=spread)
    out = call(x, V, dtype, 4)
    logp = torch.log_softmax(x.double(), 1)
    rms = lambda e: float(e.square().mean().sqrt())  # noqa: E731
    assert rms(out["lse"].double() - torch.logsumexp(x.double(), 1)) <= 2.6 * 2.0 ** -20
    assert rms(out["logprob"].double() - logp.gather(1, out["tokens"].long()[:, None])[:, 0]) <= 3.6 * 2.0 ** -20
    assert rms(out["top_logprob"].double() - logp.gather(1, out["top_id"].long())) <= 3.6 * 2.0 ** -20
    assert rms(out["entropy"].double() + (logp.exp() * logp).sum(1)) <= 4 * 2.0 ** -20
