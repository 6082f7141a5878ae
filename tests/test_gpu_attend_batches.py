"""Attention over batches that no single token stands for: the kernels of large batches, and what they leave to be joined."""
import pytest
import torch

import cache_ref as ref
from test_gpu_attend import Setup

pytestmark = pytest.mark.gpu
BF16, FP16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


@pytest.mark.parametrize("held", [BF16, E4M3])
def test_tokens_whose_positions_are_all_shared(wg, held):
    """Drafted tokens have none of their own, and their pairs are cut between blocks; sequences without a token lie between them."""
    lens = [0 if i % 5 == 2 else 700 + 13 * (i % 7) for i in range(40)]
    s = Setup(wg, lens, 8, 2, 64, held, seed=40, new=2).on_gpu()
    first = s.run(group=2)
    s.check(first)
    for _ in range(20):
        again = s.run(group=2)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])
