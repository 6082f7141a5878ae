"""A handle that was made while the default stream is busy, used at once on another stream."""
import numpy as np
import pytest
import torch

import beam_ref as ref
from test_gpu_beam import check, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


def test_new_scratch_on_another_stream(wg):
    n_req, K, V = 200, 8, 9000             # (two launches: the scan deals its items out from counters)
    x, xf, allowed, score, finished, eos = make(1, n_req, K, V, "bf16", "few", 0, K)
    want = ref.select(xf, allowed, score, finished, eos, 0, n_req, K)
    d = [t.cuda() for t in (x, torch.from_numpy(score), torch.from_numpy(finished.astype(np.int32)),
                            torch.from_numpy(ref.pack_mask(allowed).view(np.int32)))]
    so = torch.zeros((n_req, K), device="cuda")
    po, to = (torch.zeros((n_req, K), dtype=torch.int32, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(40_000_000)
    beam = wg.Beam(V, n_req, K)
    wg.wg_beam_select(beam, K, d[0], d[1], so, po, to, bitmask=d[3], finished=d[2], eos_id=eos, stream=side)
    side.synchronize()
    check((so.cpu().numpy(), po.cpu().numpy(), to.cpu().numpy()), want)
