"""Low-rank adapters where they can go wrong: the largest sizes."""
import pytest
import torch

from paper_2609_24519_b200 import binding as b

from .gpu_util import handle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,K,status", [(2 ** 31 - 1 - 65536, 64, b.OK), (2 ** 31 - 65536, 64, 2), (2 ** 31 - 1 - 4096, 64, 2), (2 ** 31 - 1, 64, 2), (2 ** 33, 64, 2),
                                        (64, 2 ** 31 - 65544, b.OK), (64, 2 ** 31 - 65536, 2), (64, 2 ** 33, 2)])
def test_sizes_whose_columns_32_bits_do_not_count(N, K, status):
    """N may be 65,536 below 2^31 - 1, so that no loop's next column wraps; a call without tokens tells whether a size is taken."""
    x = torch.zeros(64, dtype=torch.bfloat16, device="cuda")
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    got = b.OK
    try:
        b.awe_linear_adapters(handle(), b.adapters(x, x, None, b.BF16, 1, 8, N, K), x, 0, K, i, i, 1, None, N, x, b.BF16, N)
    except b.AweError as e:
        got = e.status
    assert got == status
