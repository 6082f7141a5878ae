"""Block tables at the ends of their sizes: steps without tokens, and the longest lengths."""
import numpy as np
import pytest
import torch

from test_gpu_kv import Both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


@pytest.mark.parametrize("n_seq", [1, 1024, 1025, 1500, 3000])
def test_no_tokens_at_all(wg, n_seq):
    """Nobody has a token in this step, and then some have but there is no room for them."""
    both = Both(wg, 4 * n_seq, 4, n_seq, 5)
    new = np.zeros(n_seq, np.int64)
    both.extend(new, 0)
    new[::3] = 2
    both.extend(new, 0)
    assert both.status.tolist() == [-3 if n else 0 for n in new]
    both.extend(new, int(new.sum()))
    both.extend(np.zeros(n_seq, np.int64), 0)
    assert both.lens.tolist() == new.tolist() and (both.status == 0).all()


@pytest.mark.parametrize("n_tokens", [16, 4000])
def test_lengths_up_to_32_bits(wg, n_tokens):
    """A table with room for more tokens than a length can count: the sequence ends at 2^31 - 1."""
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    block, most = 1 << 30, 2 ** 31 - 1
    pool = wg.KvPool(8, block, 3)
    pool.load(i32([1, 1, 0, 0, 0, 0, 0, 0]))
    table, lens, status = i32([[0, 1, -1, -1], [-1] * 4, [-1] * 4]), i32([most - 9, 0, 0]), i32([9] * 3)
    t = wg.KvTables(pool, table, lens, status)
    m = wg.SlotMap(3, n_tokens)
    was = table.clone()
    for too_many in (10, most):
        t.extend(i32([too_many, 0, 0]), m)
        assert status.tolist() == [-1, 0, 0] and lens.tolist() == [most - 9, 0, 0] and torch.equal(table, was)
        assert m.cu.tolist() == [0, 0, 0, 0] and (m.slot == -1).all()
    t.extend(i32([9, 0, 3]), m)
    assert status.tolist() == [0, 0, 0] and lens.tolist() == [most, 0, 3] and m.cu.tolist() == [0, 9, 9, 12]
    assert m.slot[:12].tolist() == [block + block - 10 + i for i in range(9)] + [2 * block + i for i in range(3)]
    assert m.pos[:12].tolist() == [most - 9 + i for i in range(9)] + [0, 1, 2] and (m.slot[12:] == -1).all()
    t.extend(i32([1, 0, 0]), m)
    assert status.tolist() == [-1, 0, 0] and lens.tolist() == [most, 0, 3]
    t.reorder(i32([[0, 0, 2]]))
    assert table.tolist() == [[0, 1, -1, -1], [0, 3, -1, -1], [2, -1, -1, -1]] and lens.tolist() == [most, most, 3]
    t.shrink(i32([5, most, 0]))
    assert table.tolist() == [[0, -1, -1, -1], [0, 3, -1, -1], [-1] * 4] and lens.tolist() == [5, most, 0]
    assert pool.ref.tolist() == [2, 0, 0, 1, 0, 0, 0, 0] and pool.n_free() == 6
