"""Exact attention at the far ends of its envelope: very many keys of one task."""
import math

import pytest
import torch

from paper_2607_12789_b200 import binding

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("causal", [True, False], ids=["causal", "all"])
def test_a_task_longer_than_the_limit_of_a_wait(causal):
    """One query over 50 million keys, not split: its tiles take longer than 0.2 s, which some waits of the kernel last."""
    n, d = 3 * 2 ** 24 + 77, 64
    if torch.cuda.mem_get_info()[0] < 5 * n * d * 2 // 2:
        pytest.skip("needs 16 GB of free device memory")
    # Every logit is 0 and every weight 1; sums of 1 and of -1 in tiles of 128 are exact in float32 up to 2^31, the last 77
    # keys' may be cut off by 4 (the distance of numbers about 2^25) for each of 8 groups of 16 keys: 32 / 2^25 = 2^-20.
    K, V = torch.zeros(n, 1, d, dtype=BF16, device="cuda"), torch.ones(n, 1, d, dtype=BF16, device="cuda")
    V[2 ** 25:, 0, 1] = -1
    Q = torch.ones(1, 1, d, dtype=BF16, device="cuda")
    att = binding.ExactAttention(1, 1, d, causal=causal, split=False)
    Y, L = att(Q, K, V, _ints([0, 1]), _ints([0, n]), lse=True)
    att.check()
    half = 2.0 ** -8
    want = torch.ones(d, dtype=torch.float64, device="cuda")
    want[1] = (2 ** 25 - (n - 2 ** 25)) / n
    assert ((Y[0, 0].double() - want).abs() <= 2.0 ** -20 + half * want.abs()).all()
    assert abs(L.item() - math.log(n)) <= 2.0 ** -20 + 2.0 ** -23 * math.log(n)

