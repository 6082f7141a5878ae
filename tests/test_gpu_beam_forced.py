"""Forced tokens: a row with one allowed token has probability 1 for it and keeps its score.

The logarithm of the sum is m + ln 2 * (log2 s - d), with s = 2^d as the special-function unit has it (2^-22
relative), log2 to an ulp and |d| <= 2^-13 for |m| <= 1000: off by at most 2^-21.  From |m| = 16 on that is less than
half an ulp of m (2^-21), so the result is m itself, and the score does not change at all.
"""
import numpy as np
import pytest
import torch

import beam_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wg():
    import paper_2507_16768_b200
    return paper_2507_16768_b200


@pytest.mark.parametrize("n_req,K", [(16, 8), (400, 8)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low,high,off", [(16, 1000, 0.0), (0, 16, 2.0 ** -20)])
def test_scores_of_forced_tokens_stay(wg, n_req, K, dtype, low, high, off):
    """Sixty-four steps of literals; every beam goes on with itself."""
    V, rows = 300, n_req * K
    g = torch.Generator(device="cuda").manual_seed(n_req + int(low))
    beam = wg.Beam(V, n_req, K)
    # beams in order, far enough apart to stay so
    start = -torch.arange(K, device="cuda", dtype=torch.float32).repeat(n_req)
    score = start.clone()
    parent, token = (torch.zeros((n_req, K), dtype=torch.int32, device="cuda") for _ in range(2))
    for step in range(64):
        x = low + (high - low) * torch.rand((rows, V), device="cuda", generator=g)
        x = (x * torch.where(torch.rand((rows, V), device="cuda", generator=g) < 0.5, -1.0, 1.0)).to(dtype)
        want = torch.randint(0, V, (rows,), device="cuda", generator=g, dtype=torch.int32)
        allowed = np.arange(V)[None, :] == want.cpu().numpy()[:, None]
        mask = torch.from_numpy(ref.pack_mask(allowed).view(np.int32)).cuda()
        wg.wg_beam_select(beam, K, x, score, score.view(n_req, K), parent, token, bitmask=mask)
        assert torch.equal(token.view(-1), want)
        assert torch.equal(parent, torch.arange(K, device="cuda", dtype=torch.int32).expand(n_req, K))
        # (a score of up to 8 is rounded to 2^-22 at every step where it changes at all)
        assert float((score - start).abs().max()) <= (step + 1) * (off + (2.0 ** -21 if off else 0.0)), step
