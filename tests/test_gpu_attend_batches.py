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


def check_some(s, got, window, every):
    """Every so many tokens against the 64-bit form."""
    some = torch.arange(0, s.q.shape[0], every)
    q, seq, pos = s.q, s.seq, s.pos
    s.q, s.seq, s.pos = q[some], seq[some], pos[some]
    s.check((got[0][some], got[1][some]), window)
    s.q, s.seq, s.pos = q, seq, pos


def run_and_check(s, window=0, every=7, **how):
    first = s.run(window=window, **how)
    check_some(s, first, window, every)
    empty = s.pos < 0
    assert (first[0][empty] == 0).all() and torch.isfinite(first[0].float()).all()
    again = s.run(window=window, **how)
    assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


TYPES = [(BF16, BF16), (FP16, FP16), (E4M3, BF16), (INT8, FP16)]


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("D", [64, 80, 128, 256])
@pytest.mark.parametrize("rows", [4, 12])
@pytest.mark.parametrize("window", [0, 37])
def test_warps_by_themselves(wg, held, model, D, rows, window):
    """More than 592 pairs of a token and a key head: every warp has a share of its own, over the ends of pairs."""
    lens = [(0, 1, 17, 300, 64, 5, 130)[i % 7] + i // 7 * (i % 3) for i in range(90)]
    run_and_check(Setup(wg, lens, 8 * rows, 8, D, held, model, seed=D + rows).on_gpu(), window)


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("Hq,H", [(40, 5), (96, 6), (8, 8), (128, 8), (7, 7)])
def test_warps_by_themselves_with_any_heads(wg, held, model, Hq, H):
    """Key heads that go by fours, twos and alone; one to sixteen rows of each."""
    lens = [(3, 0, 90, 16, 33)[i % 5] for i in range(150)]
    run_and_check(Setup(wg, lens, Hq, H, 64, held, model, seed=Hq).on_gpu(), every=13)


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("n", [70, 80])
def test_long_shares(wg, held, model, n):
    """Warps whose shares begin and end within long pairs."""
    run_and_check(Setup(wg, [900 + 7 * i for i in range(n)], 32, 8, 128, held, model, seed=n).on_gpu(), every=19)


@pytest.mark.parametrize("held,model", TYPES)
@pytest.mark.parametrize("D", [64, 128, 256])
def test_many_rows_are_joined_by_single_warps(wg, held, model, D):
    """More than 1184 rows and 148 pairs, drafted tokens and beams that share a prompt and have some of their own."""
    run_and_check(Setup(wg, [600 + 11 * i for i in range(40)], 16, 4, D, held, model, seed=D, new=2).on_gpu(), every=9, group=2)
    lens = [800 + 5 * i for i in range(80)]
    s = Setup(wg, lens, 16, 4, D, held, model, seed=D + 1, share={i: (i // 2 * 2, 30) for i in range(1, 80, 2)}).on_gpu()
    run_and_check(s, every=9, group=2)


@pytest.mark.parametrize("held,model", TYPES)
def test_rows_of_very_many_parts(wg, held, model):
    """One request with one key head: every block has a part of it."""
    s = Setup(wg, [30011], 4, 1, 64, held, model, seed=3).on_gpu()
    run_and_check(s, every=1)
    s = Setup(wg, [30011, 30011], 4, 1, 64, held, model, seed=4, share={1: (0, 1800)}).on_gpu()
    run_and_check(s, every=1, group=2)
