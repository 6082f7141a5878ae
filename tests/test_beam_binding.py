"""Beam search and block tables without a GPU: the binding refuses arrays that the kernels would index out of
bounds before the library is called, and the library refuses bad sizes before it touches a device."""
import ctypes

import numpy as np
import pytest
import torch

import beam_ref as ref
import paper_2507_16768_b200 as wg
from paper_2507_16768_b200 import binding
from test_binding_validation import FakeTensor


class NoLibrary:
    """Fails the test when any entry point is reached."""

    def __getattr__(self, name):
        def called(*a):
            raise AssertionError(f"{name} was called with {a}")
        return called


@pytest.fixture
def no_library(monkeypatch):
    monkeypatch.setattr(binding, "_lib", NoLibrary())


class FakeBeam:
    handle, V, device, max_out = 1, 1000, 0, 16


def plan(**k):
    R, K, C = 3, 4, 5
    args = dict(score=FakeTensor((12,), torch.float32), score_out=FakeTensor((R, C), torch.float32), parent_out=FakeTensor((R, C)),
                token_out=FakeTensor((R, C)), bitmask=FakeTensor((12, 32)), finished=FakeTensor((12,)), eos_id=2)
    return binding.BeamPlan(FakeBeam(), k.pop("n_beam", K), **dict(args, **k))


@pytest.mark.parametrize("bad", [
    dict(n_beam=0), dict(n_beam=5), dict(score=FakeTensor((12,), torch.int32)), dict(score=FakeTensor((12,), torch.float32, cuda=False)),
    dict(score=FakeTensor((24,), torch.float32, strides=(2,))), dict(score_out=FakeTensor((4, 5), torch.float32)),
    dict(score_out=FakeTensor((3, 6), torch.float32)), dict(parent_out=FakeTensor((3, 5), strides=(10, 1))),
    dict(token_out=FakeTensor((3, 5), torch.int64)), dict(bitmask=FakeTensor((12, 31))), dict(bitmask=FakeTensor((11, 32))),
    dict(bitmask=FakeTensor((12, 32), strides=(1, 12))), dict(bitmask=FakeTensor((12, 32), device=1)), dict(finished=FakeTensor((11,))),
    dict(finished=FakeTensor((12,), torch.uint8)), dict(eos_id=1000), dict(eos_id=-1), dict(token_out=FakeTensor((15,)))])
def test_a_plan_refuses(no_library, bad):
    with pytest.raises((ValueError, TypeError)):
        plan(**bad)


@pytest.mark.parametrize("bad", [FakeTensor((11, 1000), torch.float32), FakeTensor((12, 999), torch.float32), FakeTensor((12000,), torch.float32),
                                 FakeTensor((12, 1000), torch.float32, strides=(1, 12)), FakeTensor((12, 1000), torch.float32, cuda=False),
                                 FakeTensor((12, 1000), torch.float32, device=1), FakeTensor((12, 1000), torch.int32)])
def test_a_plan_refuses_logits(no_library, bad):
    p = plan()
    with pytest.raises((ValueError, TypeError)):
        p(bad)


def test_library_refuses_sizes():
    lib, h = wg.binding._lib, ctypes.c_void_p()
    for bad in ((0, 1, 1, 1), (100, 0, 1, 1), (100, 1, 0, 1), (100, 1, 33, 1), (100, 1, 1, 0), (100, 1, 1, 65), (100, 65536, 1, 1),
                (100, 3000, 32, 4), (2 ** 31 - 1, 1, 4, 4), (2 ** 30, 8, 8, 4)):
        assert lib.wg_beam_create(*bad, ctypes.byref(h)) == wg.WG_ERR_ARG and not h.value
    assert lib.wg_beam_create(100, 1, 1, 1, None) == wg.WG_ERR_ARG
    for bad in ((0, 16, 1), (-1, 16, 1), (2 ** 30 + 1, 16, 1), (10, 0, 1), (10, 2 ** 30 + 1, 1), (10, 16, 0), (10, 16, 65536)):
        assert lib.wg_kv_pool_create(*bad, ctypes.byref(h)) == wg.WG_ERR_ARG and not h.value
    assert lib.wg_kv_pool_create(10, 16, 1, None) == wg.WG_ERR_ARG
    lib.wg_beam_free(None)
    lib.wg_kv_pool_free(None)
    assert lib.wg_kv_pool_refs(None) is None


def test_plain_selection_on_a_hand_made_case():
    """Two beams, four tokens, probabilities that can be checked by hand."""
    x = np.log(np.array([[1, 2, 3, 4], [1, 1, 1, 1]], np.float64))
    allowed = np.array([[1, 0, 1, 1], [1, 1, 1, 1]], bool)
    score = np.log(np.array([0.5, 0.5], np.float32))
    got = ref.select(x, allowed, score, [False, False], 0, ref.NORM_ALLOWED, 1, 5)[0]
    # beam 0: 1/8, 3/8, 4/8; beam 1: 1/4 each; halved by the scores
    assert [(b, t) for _, b, t in got] == [(0, 3), (0, 2), (1, 0), (1, 1), (1, 2)]
    np.testing.assert_allclose(np.exp([s for s, _, _ in got]), [1 / 4, 3 / 16, 1 / 8, 1 / 8, 1 / 8], rtol=1e-6)
    got = ref.select(x, allowed, score, [False, True], 1, ref.NORM_FULL, 1, 3)[0]
    assert [(b, t) for _, b, t in got] == [(1, 1), (0, 3), (0, 2)]
    np.testing.assert_allclose(np.exp([s for s, _, _ in got]), [1 / 2, 1 / 5, 3 / 20], rtol=1e-6)


def test_plain_tables_on_a_hand_made_case():
    t = ref.Tables(6, 4, 2, 3)
    cu, slot, pos, seq, status = t.extend([5, 3], 9)
    assert cu.tolist() == [0, 5, 8] and slot.tolist() == [0, 1, 2, 3, 4, 8, 9, 10, -1] and status.tolist() == [0, 0]
    assert pos.tolist() == [0, 1, 2, 3, 4, 0, 1, 2, -1] and seq.tolist() == [0, 0, 0, 0, 0, 1, 1, 1, -1]
    copies, src, dst, status = t.reorder(np.array([[0, 0]]))
    assert copies == [(1, 2, 1)] and t.rows == [[0, 1], [0, 2]] and t.ref == [2, 1, 1, 0, 0, 0] and t.len == [5, 5]
    t.shrink([4, 0])
    assert t.rows == [[0], []] and t.ref == [1, 0, 0, 0, 0, 0]


def test_plain_backtrack_on_a_hand_made_case():
    token = np.array([[[1, 2]], [[3, 4]], [[5, 6]]], np.int32)
    parent = np.array([[[0, 0]], [[1, 0]], [[0, -1]]], np.int32)
    assert ref.backtrack(token, parent).tolist() == [[[2, 3, 5], [-1, -1, -1]]]
