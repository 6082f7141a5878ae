"""Steps without a token (all beams have ended, say): arrays without elements have no address, and nothing is to be done."""
import pytest
import torch

import paper_2507_16768_b200 as wg
from test_beam_binding import FakeTensor
from test_cache_binding import At, FakeSlots, cache, lib_write, on_device_zero, other, write  # noqa: F401


@pytest.mark.parametrize("heads", [0, 8])
def test_the_library_writes_no_tokens(heads):
    nothing = dict(n=0, k=None, v=None, slot=None, pos=None)
    assert lib_write(q=None, o=None, heads=heads, **nothing) == wg.WG_OK
    assert lib_write(heads=heads, **nothing) == wg.WG_OK
    assert lib_write(q=None, o=None, heads=heads, rope_=None, **nothing) == wg.WG_OK
    for bad in (dict(heads=-1), dict(heads=70000), dict(dtype=1), dict(rope_=dict(rot_dim=8))):
        assert lib_write(**dict(nothing, **bad)) == wg.WG_ERR_ARG


def test_the_binding_writes_no_tokens():
    slots = other(FakeSlots, n_tokens=0, _args=(0x1000, None, None, None, 0))
    for storage in (torch.bfloat16, torch.int8):
        k, q = At((0, 2, 64), at=0), At((0, 8, 64), at=0)
        for how in (dict(q=q, q_out=None), dict(q=q, q_out=q), dict(q=None, q_out=None), dict(q=q, q_out=None, rope=None),
                    dict(q=q, q_out=None, status=FakeTensor((0,)))):
            write(cache(storage), k=k, v=k, slots=slots, **dict(dict(rope=None), **how))
