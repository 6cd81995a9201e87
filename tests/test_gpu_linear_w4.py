"""The linear layer with 4-bit weights against its definition in 64 bits.

Tolerance.  Products are exact; with S = sum_k |x| |scale| |code - zero| the FP32 sums over the matrix steps of a group
(at most 16), over the groups and over at most 8 parts of K are off by at most (16 + groups + 10) 2^-22 S, and y is rounded once
with the unit roundoff u of its type: |y - ref| <= u |ref| + (26 + groups) 2^-22 S (+ the smallest FP16 step).
"""
import numpy as np
import pytest
import torch

from paper_2609_24519_b200 import binding as b
from tests.gpu_util import handle

pytestmark = pytest.mark.gpu

TYPES = {"f16": (b.F16, torch.float16, 2.0 ** -11), "bf16": (b.BF16, torch.bfloat16, 2.0 ** -8), "f32": (b.F32, torch.float32, 2.0 ** -23)}


def pack(q, ld):
    """N x K values in [-8, 7] -> rows of ld / 2 bytes, low nibble first; what lies behind K is not zero."""
    N, K = q.shape
    wide = np.full((N, ld), 5, np.int64)
    wide[:, :K] = q
    return ((wide[:, 0::2] & 15) | (wide[:, 1::2] & 15) << 4).astype(np.uint8)


def check(M, N, K, group, x_kind="f16", y_kind="f16", s_kind=None, zero=False, ld=None, offset=0, ldx_extra=0, ldy_extra=0, x_offset=0, x=None):
    s_kind = s_kind or x_kind
    rng = np.random.default_rng(M * 7 + N + K + group)
    ld = ld or -(-K // 32) * 32
    groups = -(-K // group)
    q = rng.integers(-8, 8, (N, K))
    scale = torch.from_numpy((rng.random((N, groups)) * 0.1 + 0.01).astype(np.float32)).to(TYPES[s_kind][1])
    z = rng.integers(-8, 8, (N, groups)) if zero else np.zeros((N, groups), int)
    if x is None:
        x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).to(TYPES[x_kind][1])
    codes = torch.zeros(N * ld // 2 + offset, dtype=torch.uint8, device="cuda")
    codes[offset:] = torch.from_numpy(pack(q, ld).reshape(-1)).cuda()
    dx = torch.full((M * (K + ldx_extra) + x_offset,), float("nan"), dtype=x.dtype, device="cuda")  # nothing between rows is read
    dx[x_offset:].view(M, K + ldx_extra)[:, :K] = x.cuda()
    y = torch.full((M, N + ldy_extra), 77.0, dtype=TYPES[y_kind][1], device="cuda")
    junk = torch.from_numpy((z & 15) | 0x50).to(torch.int8).cuda() if zero else None  # only the low nibble counts
    W = b.w4_matrix(codes[offset:], scale.cuda(), TYPES[s_kind][0], junk, N, K, ld, group)
    outs = []
    for _ in range(2):
        y.fill_(77.0)
        b.awe_linear_w4(handle(), W, dx[x_offset:], TYPES[x_kind][0], M, K + ldx_extra, y, TYPES[y_kind][0], N + ldy_extra)
        torch.cuda.synchronize()
        outs.append(y.clone())
    assert torch.equal(outs[0], outs[1]) and bool((y[:, N:] == 77).all())
    g = np.arange(K) // group
    w = scale.double().numpy()[:, g] * (q - z[:, g])
    ref, S = x.double().numpy() @ w.T, np.abs(x.double().numpy()) @ np.abs(w).T
    got = y[:, :N].double().cpu().numpy()
    tol = TYPES[y_kind][2] * np.abs(ref) + (26 + groups) * 2.0 ** -22 * S + (2.0 ** -25 if y_kind == "f16" else 0)
    assert (np.abs(got - ref) <= tol).all(), float(np.max(np.abs(got - ref) - tol))


@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("x_kind,y_kind", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32")])
def test_rows_of_x(M, x_kind, y_kind):
    check(M, 200, 1000, 128, x_kind, y_kind, zero=M % 2 == 0)


@pytest.mark.parametrize("N", [1, 15, 63, 64, 65, 130, 1000])
@pytest.mark.parametrize("K", [1, 31, 32, 33, 255, 257, 2049, 5000])
def test_odd_sizes(N, K):
    check(3, N, K, 64, zero=True)


@pytest.mark.parametrize("group", [32, 64, 128, 256, 512, 8192, 1 << 20])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("M", [1, 40])
def test_groups(group, zero, M):
    check(M, 100, 3333, group, "bf16", "f32", "f16", zero)


@pytest.mark.parametrize("M", [1, 5, 20, 77])
@pytest.mark.parametrize("ld,offset,ldx_extra,x_offset,ldy_extra", [(1002, 0, 0, 0, 0), (1024, 1, 0, 0, 0), (1006, 3, 3, 1, 5), (1056, 16, 8, 8, 8), (1002, 15, 0, 7, 1)])
def test_strides_and_alignments(M, ld, offset, ldx_extra, x_offset, ldy_extra):
    check(M, 90, 1001, 32, "f16", "f16", zero=True, ld=ld, offset=offset, ldx_extra=ldx_extra, x_offset=x_offset, ldy_extra=ldy_extra)


def test_long_rows():
    check(2, 70, 70000, 128, "bf16", "bf16", zero=True)
    check(150, 130, 20011, 64, "f16", "f32")


def test_an_infinity_stays_in_its_row():
    x = torch.ones((20, 300), dtype=torch.float16)
    x[3, 7], x[4, 299] = float("inf"), float("nan")
    codes = torch.full((50, 160), 0x11, dtype=torch.uint8, device="cuda")  # every code is 1
    W = b.w4_matrix(codes, torch.ones((50, 10), dtype=torch.float16, device="cuda"), b.F16, None, 50, 300, 320, 32)
    y = torch.zeros((20, 50), dtype=torch.float16, device="cuda")
    b.awe_linear_w4(handle(), W, x.cuda(), b.F16, 20, 300, y, b.F16, 50)
    y = y.cpu()
    assert bool(torch.isposinf(y[3]).all()) and bool(torch.isnan(y[4]).all())
    rest = [i for i in range(20) if i not in (3, 4)]
    assert bool((y[rest] == 300).all())


def test_refusals():
    INVALID, UNSUPPORTED, ALIGNMENT = 1, 2, 4
    h = handle()
    d = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    at = d.data_ptr()

    def linear(x=at, x_t=b.F16, M=2, ldx=64, y=at, y_t=b.F16, ldy=8, raw=None, **kw):
        W = b.W4Matrix(**{**dict(codes_dev=at, scale_dev=at, zero_dev=0, N=8, K=64, ld=64, group=32, scale_type=b.F16), **kw})
        return b.lib().awe_linear_w4(h.raw if raw is None else None, W, x, x_t, M, ldx, y, y_t, ldy, None)

    launches = b.awe_launch_count(h)
    for bad in (dict(raw=0), dict(x=0), dict(y=0), dict(M=-1), dict(ldx=63), dict(ldy=7), dict(x_t=5), dict(y_t=-1), dict(codes_dev=0), dict(scale_dev=0),
                dict(N=0), dict(K=0), dict(ld=62), dict(ld=65), dict(scale_type=3)):
        assert linear(**bad) == INVALID, bad
    for bad in (dict(x_t=b.F32), dict(y_t=b.BF16), dict(scale_type=b.F32), dict(group=16), dict(group=48), dict(group=0)):
        assert linear(**bad) == UNSUPPORTED, bad
    for bad in (dict(x=at + 1), dict(y=at + 1), dict(scale_dev=at + 1), dict(y=at + 2, y_t=b.F32)):
        assert linear(**bad) == ALIGNMENT, bad
    assert linear(M=0, x=0) == 0
    assert b.awe_launch_count(h) == launches
