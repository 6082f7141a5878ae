"""Attention over 8-bit caches whose values have scales of any size, none, or no number."""
import math

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


def same_tables(lens):
    """All sequences on the first columns of the longest."""
    longest = lens.index(max(lens))
    return {i: (longest, -(-n // 16)) for i, n in enumerate(lens) if i != longest}


def check_lse(s, lse, window=0, scale=None):
    """The scores' sum has no values in it: as with values of 1."""
    scale = s.scale if scale is None else scale
    ones = torch.ones(s.v.shape, dtype=torch.float64)
    want, want_lse, mass, size = ref.attend(s.q, ref.held(s.k, s.ks), ones, s.table, s.seq, s.pos, scale, window)
    # (every scale counts as 2^-80 at least: an exponent of 80 and a step of it)
    _, tol = ref.tolerance(want, mass, size, (s.pos + 1).clamp(min=1), s.D, s.model, FP16, torch.tensor([2.0 ** -80]))
    empty = want_lse == -math.inf
    assert (lse[empty] == -math.inf).all()
    off = (lse.double() - want_lse)[~empty].abs()
    assert (off <= tol.expand_as(want_lse)[~empty]).all(), off.max().item()


def far_below(s):
    """Scores of about -240, all alike."""
    s.q.zero_()
    s.q[..., 0] = -400.0
    s.k.zero_()
    s.k[..., 0] = torch.tensor(96.0).to(s.held)
    s.ks.fill_(0.05)
    s.scale = 0.125


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("low", [False, True])
@pytest.mark.parametrize("window", [0, 1])
@pytest.mark.parametrize("lens", [[1, 40, 0, 300, 2500], [1 + i % 70 for i in range(80)]])
def test_values_without_a_number(wg, held, model, low, window, lens):
    """No visible value has one: every result is NaN, and the scores' sum is what it is."""
    for share in (None, same_tables(lens)):
        s = Setup(wg, lens, 8, 2, 64, held, model, seed=1, share=share)
        if low:
            far_below(s)
        s.vs.fill_(math.nan)
        s.on_gpu()
        for group in (1, 5):
            out, lse = s.run(window=window, group=group, scale=s.scale)
            some = s.lens > 0
            assert torch.isnan(out[some]).all() and (out[~some] == 0).all()
            check_lse(s, lse, window)


@pytest.mark.parametrize("held,model", [(E4M3, BF16), (INT8, FP16)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("lens", [[1, 40, 0, 300, 2500], [1 + i % 70 for i in range(80)]])
def test_a_value_without_a_number(wg, held, model, bad, lens):
    """One of each sequence's, of the first head: NaN everywhere, or infinite where its code is not 0."""
    for share in (None, same_tables(lens)):
        s = Setup(wg, lens, 8, 2, 64, held, model, seed=2, share=share)
        clean = Setup(wg, lens, 8, 2, 64, held, model, seed=2, share=share).on_gpu()
        at = {}
        for i, n in enumerate(lens):
            if n:
                p = (0 if share else 3 * n // 4)
                at[i] = (int(s.table[i, p // 16]), p % 16)
                s.vs[at[i]][0] = bad
        s.on_gpu()
        for group in (1, 5):
            (out, lse), (want, _) = s.run(group=group), clean.run(group=group)
            check_lse(s, lse)
            for i, (b, o) in at.items():
                code = s.v[b, o, 0].float()
                first = torch.where(code == 0, math.nan, torch.sign(code) * bad).expand(4, -1)
                assert torch.equal(torch.isnan(out[i, :4]), torch.isnan(first))
                assert torch.equal(out[i, :4].float()[~torch.isnan(first)], first[~torch.isnan(first)])
                assert torch.equal(out[i, 4:], want[i, 4:])


@pytest.mark.parametrize("held", [E4M3, INT8])
def test_values_of_infinite_scale_alone(wg, held):
    """Tokens that see one position, and tokens that see nothing else."""
    lens = [1, 1, 30, 2000]
    s = Setup(wg, lens, 8, 2, 64, held, BF16, seed=3)
    s.vs.fill_(math.inf)
    s.v.fill_(2.0) if held is E4M3 else s.v.fill_(2)
    s.v[..., 1::2] = torch.tensor(-3.0).to(held)
    s.on_gpu()
    for group in (1, 2):
        out, lse = s.run(group=group)
        assert (out[..., 0::2] == math.inf).all() and (out[..., 1::2] == -math.inf).all()
        check_lse(s, lse)
