"""Steps without a token on the GPU: nothing is written, attended to or read, and nothing is refused."""
import os
import sys

import pytest
import torch

import paper_2507_16768_b200 as wg
from wg_workloads import make_vocab

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("held", [torch.bfloat16, torch.float8_e4m3fn])
def test_a_step_of_no_tokens(held):
    c = wg.KvCache.empty(2, 16, 2, 64, held)
    before = c.keys.view(torch.uint8).clone()
    slots, rope = wg.SlotMap(3, 0), wg.Rope(10, 64)
    k, q = (torch.empty((0, h, 64), dtype=torch.bfloat16, device="cuda") for h in (2, 8))
    status = torch.empty(0, dtype=torch.int32, device="cuda")
    for how in (dict(q=q), dict(q=q, q_out=torch.empty_like(q)), dict(q=q, rope=rope), dict(q=q, rope=rope, status=status)):
        c.write(k, k, slots, **how)
    pool = wg.KvPool(2, 16, 3)
    tables = wg.KvTables(pool, torch.full((3, 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))
    tables.extend(torch.zeros(3, dtype=torch.int32, device="cuda"), slots)
    wg.Attend(4, 8, 2, 64)(q, c, tables, torch.empty_like(q), slots=slots)
    c.read(tables, torch.zeros(4, dtype=torch.int32, device="cuda"), k, k)
    torch.cuda.synchronize()
    assert torch.equal(c.keys.view(torch.uint8), before)


def test_the_example_goes_on_when_all_beams_have_ended():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import beam_search as ex
    vocab = make_vocab(2000, seed=1)
    model = ex.ToyModel(vocab)
    own = ex.LibraryCache(4, 40, 16, 2)
    none = torch.zeros(4, dtype=torch.int32, device="cuda")
    own.append(torch.tensor([3, 0, 2, 0], dtype=torch.int32, device="cuda"), torch.arange(5, device="cuda"), model)
    want = own.attend()
    own.append(none, torch.empty(0, dtype=torch.int64, device="cuda"), model)
    assert torch.equal(own.attend(), want)
