"""The layer operators at the ends of what they take."""
import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


# few tokens, k split over 16 and 4 parts and joined, tiles alone
@pytest.mark.parametrize("T,m", [(3, 5), (40, 5), (70, 5), (1000, 1000), (2048, 2048)])
def test_q8_sums_of_two_to_the_31(gpu, T, m):
    """131072 products of (-128)^2 are 2^31 exactly, one more than 32 bits hold."""
    n = 131072
    q = torch.full((T, n), -128, dtype=torch.int8, device=gpu)
    Z = torch.full((m, n), -128, dtype=torch.int8, device=gpu)
    q[1] = 127
    Z[2] = 127
    q[T - 1, n - 1] = -127
    y = ffe.linear_q8(q, torch.ones(T, device=gpu), Z, torch.ones(m, device=gpu))
    rows, cols = torch.full((T,), -128.0, dtype=torch.float64), torch.full((m,), -128.0, dtype=torch.float64)
    rows[1], cols[2] = 127, 127
    want = rows[:, None] * cols * n
    want[T - 1] += cols
    assert torch.equal(y.cpu(), want.to(BF16))
