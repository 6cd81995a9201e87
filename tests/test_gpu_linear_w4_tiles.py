"""The 4-bit linear layer on each of its tcgen05 tiles and on both sides of the rules that choose.

Sizes that no tile divides, codes and rows of x at any alignment, K in one part and in several.  The definition, the tolerance and
the poisoned gaps between rows are those of test_gpu_linear_w4.check.
"""
import pytest

from tests.test_gpu_linear_w4 import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [9, 16, 17, 33, 65, 100, 128, 129, 200, 300])
@pytest.mark.parametrize("N", [2049, 5003])
@pytest.mark.parametrize("K", [333, 800])
def test_ragged_sizes(M, N, K):
    check(M, N, K, 32 if K == 333 else 128, "bf16" if M % 2 else "f16", "f32" if N == 2049 else ("bf16" if M % 2 else "f16"), zero=K == 333)


@pytest.mark.parametrize("M", [16, 30, 64, 128, 139])
@pytest.mark.parametrize("ld,offset,ldx_extra,x_offset,ldy_extra", [(1002, 0, 0, 0, 0), (1024, 1, 0, 0, 0), (1006, 3, 3, 1, 5), (1056, 16, 7, 8, 8), (1002, 15, 0, 7, 1)])
def test_strides_and_alignments(M, ld, offset, ldx_extra, x_offset, ldy_extra):
    check(M, 4300, 1001, 32, "f16", "f16", zero=True, ld=ld, offset=offset, ldx_extra=ldx_extra, x_offset=x_offset, ldy_extra=ldy_extra)


@pytest.mark.parametrize("M,N", [(12, 2100), (24, 300), (64, 300), (128, 300), (70, 4200), (150, 4200)])
@pytest.mark.parametrize("K,ld,x_offset", [(4096, 4096, 0), (4097, 4098, 0), (5000, 5024, 1), (8191, 8192, 3)])
def test_long_rows(M, N, K, ld, x_offset):
    """Rings that go round, more than one slab of scales, K in one part and in several."""
    check(M, N, K, 64, "bf16", "f32", zero=True, ld=ld, x_offset=x_offset)


@pytest.mark.parametrize("group", [32, 64, 128, 256, 512, 1 << 20])
@pytest.mark.parametrize("zero", [False, True])
@pytest.mark.parametrize("M,N,ld", [(14, 2065, 2080), (14, 2065, 2050), (101, 4200, 2080), (101, 4200, 2050)])
def test_groups(group, zero, M, N, ld):
    check(M, N, 2049, group, "f16", "f16", "bf16", zero, ld=ld)


@pytest.mark.parametrize("M,N,K", [(17, 4100, 8001), (32, 7000, 2101), (33, 2501, 6001), (64, 2049, 3601), (65, 2049, 3501), (100, 1500, 3201),
                                   (65, 4300, 1701), (128, 4224, 900), (139, 4200, 801), (300, 5003, 333)])
@pytest.mark.parametrize("codes_aligned", [True, False])
@pytest.mark.parametrize("x_aligned", [True, False])
def test_products_that_are_worth_tcgen05(M, N, K, codes_aligned, x_aligned):
    """From 4.5e8 on: the tiles of 32, 64 and 128 rows, codes and x with and without TMA."""
    assert M * N * K >= 4.5e8
    kinds = {True: ("f16", "f16"), False: ("bf16", "f32")}[x_aligned]
    ld = (K + 31) // 32 * 32 if codes_aligned else K + K % 2 + 2
    check(M, N, K, {0: 32, 1: 64, 2: 128, 3: 256}[(M + K + codes_aligned) % 4], *kinds, zero=codes_aligned != x_aligned, ld=ld, offset=0 if codes_aligned else 3,
          ldx_extra=-K % 8 if x_aligned else 1 - K % 2, x_offset=0 if x_aligned else 1)
