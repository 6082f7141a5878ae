"""Beam-search and block-table calls refuse arrays of a device that is not the current one (no GPU needed: stand-ins for
tensors, and a library that fails the test when it is reached)."""
import pytest
import torch

from paper_2507_16768_b200 import binding
from test_beam_binding import FakeBeam, no_library, plan  # noqa: F401
from test_binding_validation import FakeTensor


@pytest.fixture
def current(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    return lambda device: monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: device, raising=False)


class FakePool:
    handle, n_blocks, block_size, max_seqs, device = 1, 16, 4, 8, 0


class FakeSlots:
    n_seq, device, _args = 4, 0, (1, 1, 1, 1, 8)


class FakeContext:
    handle, device = 1, 0

    class vocab:
        V, W = 1000, 32


def calls():
    i32 = FakeTensor
    tables = binding.KvTables(FakePool(), i32((4, 5)), i32((4,)), i32((4,)))
    pool = binding.KvPool.__new__(binding.KvPool)
    pool.handle, pool.n_blocks, pool.device = 1, 16, 0
    f32 = lambda *shape: FakeTensor(shape, torch.float32)  # noqa: E731
    select = plan()
    return [
        lambda: select(f32(12, 1000)),
        lambda: binding.wg_beam_step(FakeBeam(), FakeContext(), 4, i32((12,)), i32((12,)), f32(12), f32(12, 1000), i32((12, 32)),
                                     i32((12,)), i32((12,))),
        lambda: binding.wg_beam_backtrack(i32((5, 3, 4)), i32((5, 3, 4)), i32((3, 4, 5))),
        lambda: tables.extend(i32((4,)), FakeSlots()),
        lambda: tables.shrink(i32((4,))),
        lambda: tables.reorder(i32((2, 2))),
        lambda: pool.load(i32((16,))),
        lambda: pool.n_free(),
    ]


def test_the_current_device_is_taken(no_library, current):  # noqa: F811
    current(0)
    for call in calls():
        with pytest.raises(AssertionError, match="was called"):
            call()


def test_another_device_is_refused(no_library, current):  # noqa: F811
    current(1)
    for call in calls():
        with pytest.raises(ValueError, match="not the current device"):
            call()


def test_scratch_of_another_device_is_refused(no_library, current):  # noqa: F811
    current(0)

    class Elsewhere(FakeBeam):
        device = 1
    f32 = lambda *shape: FakeTensor(shape, torch.float32)  # noqa: E731
    with pytest.raises(ValueError, match="scratch"):
        binding.wg_beam_step(Elsewhere(), FakeContext(), 4, FakeTensor((12,)), FakeTensor((12,)), f32(12), f32(12, 1000),
                             FakeTensor((12, 32)), FakeTensor((12,)), FakeTensor((12,)))
