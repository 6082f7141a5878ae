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
