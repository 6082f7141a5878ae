"""What a paged cache holds, without a GPU: the binding refuses arrays that the kernels would index out of bounds before the
library is called, the library refuses bad sizes and pointers before it touches a device, and the angles' frequencies."""
import ctypes as C

import numpy as np
import pytest
import torch

import cache_ref as ref
import paper_2507_16768_b200 as wg
from paper_2507_16768_b200 import binding
from test_beam_binding import no_library  # noqa: F401
from test_binding_validation import FakeTensor

BF16, FP16, FP32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(autouse=True)
def on_device_zero(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)


class At(FakeTensor):
    """A stand-in at a given address."""

    def __init__(self, shape, dtype=BF16, at=0x1000, **k):
        super().__init__(shape, dtype, **k)
        self.at = at

    def data_ptr(self):
        return self.at

    def stride(self, *i):
        return super().stride(*i) if i else self._strides

    def get_device(self):
        return self.device.index if self.is_cuda else -1


def cache(dtype=BF16, n_blocks=8, block=4, H=2, D=64, **k):
    planes = dict(keys=At((n_blocks, block, H, D), dtype), values=At((n_blocks, block, H, D), dtype))
    if dtype in (E4M3, torch.int8):
        planes.update(key_scale=At((n_blocks, block, H), FP32), value_scale=At((n_blocks, block, H), FP32))
    planes.update(k)
    return binding.KvCache(**planes)


@pytest.mark.parametrize("bad", [
    dict(values=At((8, 4, 2, 64), FP16)), dict(values=At((8, 4, 2, 32))), dict(keys=At((8, 4, 2, 64), FP32)), dict(keys=At((8, 4, 128))),
    dict(values=At((8, 4, 2, 64), at=0x1008)), dict(values=At((8, 4, 2, 64), device=1)), dict(values=At((8, 4, 2, 64), cuda=False)),
    dict(values=At((8, 4, 2, 64), strides=(1024, 128, 64, 1))), dict(key_scale=At((8, 4, 2), FP32), value_scale=At((8, 4, 2), FP32)),
    dict(key_scale=At((8, 4, 2), FP32))])
def test_a_cache_refuses(bad):
    with pytest.raises((ValueError, TypeError)):
        cache(**bad)


@pytest.mark.parametrize("shape", [(8, 4, 2, 8), (8, 4, 2, 72), (8, 4, 2, 272), (0, 4, 2, 64), (8, 0, 2, 64), (8, 4, 0, 64)])
def test_a_cache_refuses_sizes(shape):
    with pytest.raises(ValueError):
        binding.KvCache(At(shape), At(shape))


@pytest.mark.parametrize("bad", [dict(key_scale=None), dict(value_scale=None), dict(key_scale=At((8, 4, 2), BF16)), dict(value_scale=At((8, 4), FP32)),
                                 dict(value_scale=At((8, 4, 2), FP32, device=1)), dict(value_scale=At((8, 4, 2), FP32, strides=(1, 8, 32)))])
def test_an_8_bit_cache_refuses(bad):
    with pytest.raises((ValueError, TypeError)):
        cache(E4M3, **bad)


class FakeSlots:
    n_seq, n_tokens, device, _args = 4, 6, 0, (0x1000,) * 4 + (6,)


class FakePool:
    handle, n_blocks, block_size, max_seqs, device = 1, 8, 4, 8, 0


class FakeRope:
    rot_dim, device, _arg = 64, 0, 0x1000


def other(cls, **k):
    return type("Other", (cls,), k)()


def write(c=None, **k):
    args = dict(k=At((6, 2, 64)), v=At((6, 2, 64)), slots=FakeSlots(), rope=FakeRope(), q=At((6, 8, 64)), q_out=At((6, 8, 64)))
    args.update(k)
    (c or cache()).write(**args)


def test_a_good_write_reaches_the_library(no_library):  # noqa: F811
    strided = dict(k=At((6, 2, 64), strides=(1024, 64, 1)), q_out=None)
    for how in ({}, strided, dict(q=None, q_out=None), dict(rope=None, q=None, q_out=None), dict(rope=None), dict(status=FakeTensor((6,)))):
        with pytest.raises(AssertionError, match="wg_kv_write was called"):
            write(**how)
    with pytest.raises(AssertionError, match="wg_kv_write was called"):
        write(cache(E4M3))


@pytest.mark.parametrize("bad", [
    dict(k=At((5, 2, 64))), dict(k=At((6, 2, 32))), dict(k=At((6, 4, 64))), dict(k=At((6, 128))), dict(k=At((6, 2, 64), FP32)), dict(k=At((6, 2, 64), FP16)),
    dict(v=At((6, 2, 64), FP16)), dict(v=At((6, 2, 64), device=1)), dict(v=At((6, 2, 64), cuda=False)), dict(v=At((6, 2, 64), at=0x1002)),
    dict(v=At((6, 2, 64), strides=(132, 64, 1))), dict(v=At((6, 2, 64), strides=(64, 64, 1))), dict(v=At((6, 2, 64), strides=(0, 64, 1))),
    dict(v=At((6, 2, 64), strides=(128, 1, 2))), dict(v=At((6, 2, 64), strides=(256, 128, 1))), dict(q=At((7, 8, 64))), dict(q=At((6, 0, 64))),
    dict(q=At((6, 512))), dict(q_out=At((6, 4, 64))), dict(q_out=At((6, 8, 64), FP16)), dict(q=None),
    dict(slots=other(FakeSlots, device=1)), dict(slots=other(FakeSlots, n_tokens=7)), dict(rope=other(FakeRope, device=1)),
    dict(rope=other(FakeRope, rot_dim=80)), dict(status=FakeTensor((5,))), dict(status=FakeTensor((6,), torch.int64))])
def test_a_write_refuses(no_library, bad):  # noqa: F811
    with pytest.raises((ValueError, TypeError)):
        write(**bad)


def tables(n_seq=4, **k):
    pool = other(FakePool, **k)
    return binding.KvTables(pool, FakeTensor((n_seq, 5)), FakeTensor((n_seq,)))


def read(c=None, t=None, **k):
    args = dict(cu=FakeTensor((5,)), k_out=At((9, 2, 64)), v_out=At((9, 2, 64)))
    args.update(k)
    (c or cache()).read(t or tables(), **args)


def test_a_good_read_reaches_the_library(no_library):  # noqa: F811
    for how in ({}, dict(k_out=None), dict(v_out=None), dict(k_out=At((9, 2, 64), FP32), v_out=None)):
        with pytest.raises(AssertionError, match="wg_kv_read was called"):
            read(**how)


@pytest.mark.parametrize("bad", [
    dict(cu=FakeTensor((4,))), dict(cu=FakeTensor((5,), torch.int64)), dict(k_out=None, v_out=None), dict(k_out=At((8, 2, 64))),
    dict(k_out=At((9, 2, 64), FP32)), dict(k_out=At((9, 2, 64), torch.int32), v_out=None), dict(k_out=At((9, 2, 64), at=0x1004)),
    dict(k_out=At((9, 2, 64), strides=(256, 64, 1))), dict(k_out=At((9, 2, 64), cuda=False)), dict(v_out=At((9, 2, 64), device=1)),
    dict(v_out=At((9, 1, 64)), k_out=None), dict(t=tables(block_size=8)), dict(t=tables(n_blocks=9)), dict(t=tables(device=0, n_blocks=9))])
def test_a_read_refuses(no_library, bad):  # noqa: F811
    with pytest.raises((ValueError, TypeError)):
        read(**bad)


class FakeAttend:
    handle, max_tokens, n_q_heads, n_heads, head_dim, device, scale = 1, 8, 8, 2, 64, 0, 0.125


def attend(a=None, c=None, t=None, **k):
    args = dict(q=At((4, 8, 64)), out=At((4, 8, 64)))
    args.update(k)
    binding.Attend.__call__(a or FakeAttend(), args.pop("q"), c or cache(), t or tables(), **args)


def test_a_good_attention_reaches_the_library(no_library):  # noqa: F811
    six = dict(q=At((6, 8, 64)), out=At((6, 8, 64)), slots=FakeSlots())
    for how in ({}, six, dict(lse=At((4, 8), FP32)), dict(q=At((3, 8, 64)), out=At((3, 8, 64))), dict(c=cache(E4M3)),
                dict(c=cache(E4M3), q=At((4, 8, 64), FP16), out=At((4, 8, 64), FP16))):
        with pytest.raises(AssertionError, match="wg_kv_attend was called"):
            attend(**how)


@pytest.mark.parametrize("bad", [
    dict(q=At((5, 8, 64))), dict(q=At((4, 4, 64))), dict(q=At((4, 8, 64), FP16)), dict(q=At((4, 8, 64), FP32)), dict(out=At((3, 8, 64))),
    dict(out=At((4, 8, 64), FP16)), dict(out=At((4, 8, 64), at=0x1008)), dict(out=At((4, 8, 64), strides=(516, 64, 1))), dict(lse=At((4, 8))),
    dict(lse=At((4, 2), FP32)), dict(lse=At((4, 8), FP32, strides=(16, 1))), dict(lse=At((4, 8), FP32, cuda=False)), dict(slots=FakeSlots()),
    dict(slots=other(FakeSlots, device=1), q=At((6, 8, 64)), out=At((6, 8, 64))), dict(slots=other(FakeSlots, n_seq=5), q=At((6, 8, 64)), out=At((6, 8, 64))),
    dict(a=other(FakeAttend, max_tokens=3)), dict(a=other(FakeAttend, device=1)), dict(a=other(FakeAttend, n_heads=4)),
    dict(a=other(FakeAttend, head_dim=128)), dict(t=tables(block_size=8)), dict(t=tables(n_blocks=9))])
def test_an_attention_refuses(no_library, bad):  # noqa: F811
    with pytest.raises((ValueError, TypeError)):
        attend(**bad)


def test_another_device_is_refused(no_library, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1, raising=False)
    for call in (write, read, attend):
        with pytest.raises(ValueError, match="not the current device"):
            call()


# ---- the library itself ------------------------------------------------------------------------------------------
lib = wg.binding._lib


def struct(**k):
    fields = dict(k=0x1000, v=0x1000, k_scale=None, v_scale=None, storage=0, n_blocks=8, block_size=4, n_heads=2, head_dim=64)
    fields.update(k)
    return binding._WgKvCache(**fields)


def rope(**k):
    fields = dict(table=0x1000, n_pos=10, rot_dim=64, interleaved=0)
    fields.update(k)
    return binding._WgRope(**fields)


BAD_CACHES = [dict(k=None), dict(v=None), dict(k=0x1008), dict(storage=4), dict(storage=-1), dict(storage=2), dict(k_scale=0x1000, v_scale=0x1000),
              dict(storage=3, k_scale=0x1000), dict(storage=3, k_scale=0x1002, v_scale=0x1000), dict(n_blocks=0), dict(n_blocks=2 ** 30 + 1),
              dict(block_size=0), dict(block_size=2 ** 30 + 1), dict(n_heads=0), dict(n_heads=1025), dict(head_dim=0), dict(head_dim=24),
              dict(head_dim=272)]


def lib_write(cache_=None, k=0x1000, ks=128, v=0x1000, vs=128, q=0x1000, qs=512, o=0x1000, os=512, heads=8, dtype=0, rope_=(), slot=0x1000, pos=0x1000,
              n=4, status=None):
    c, r = struct(**(cache_ or {})), None if rope_ is None else rope(**dict(rope_))
    return lib.wg_kv_write(C.addressof(c), k, ks, v, vs, q, qs, o, os, heads, dtype, None if r is None else C.addressof(r), slot, pos, n, status, None)


@pytest.mark.parametrize("bad", [dict(cache_=c) for c in BAD_CACHES] + [
    dict(n=-1), dict(heads=-1), dict(heads=0), dict(heads=70000), dict(dtype=1), dict(dtype=2), dict(dtype=3), dict(q=None), dict(o=None),
    dict(rope_=dict(table=None)), dict(rope_=dict(table=0x1004)), dict(rope_=dict(n_pos=0)), dict(rope_=dict(rot_dim=8)), dict(rope_=dict(rot_dim=24)),
    dict(rope_=dict(rot_dim=80)), dict(k=None), dict(v=None), dict(k=0x1002), dict(ks=120), dict(ks=132), dict(vs=64), dict(qs=504), dict(os=508),
    dict(q=0x1008), dict(slot=None), dict(pos=None)])
def test_library_refuses_writes(bad):
    assert lib_write(**bad) == wg.WG_ERR_ARG
    assert lib.wg_kv_write(None, *[None, 0] * 4, 0, 0, None, None, None, 0, None, None) == wg.WG_ERR_ARG


def lib_read(cache_=None, table=0x1000, stride=5, cols=5, lens=0x1000, n_seq=4, cu=0x1000, k=0x1000, v=0x1000, dtype=0, rows=10):
    c = struct(**(cache_ or {}))
    return lib.wg_kv_read(C.addressof(c), table, stride, cols, lens, n_seq, cu, k, v, dtype, rows, None)


@pytest.mark.parametrize("bad", [dict(cache_=c) for c in BAD_CACHES] + [
    dict(table=None), dict(stride=4), dict(cols=0), dict(lens=None), dict(n_seq=0), dict(cu=None), dict(k=0x1008), dict(v=0x1004), dict(dtype=3),
    dict(dtype=-1), dict(rows=-1)])
def test_library_refuses_reads(bad):
    assert lib_read(**bad) == wg.WG_ERR_ARG


def test_calls_without_work_do_nothing():
    assert lib_write(n=0, k=None, v=None, q=None, o=None, heads=0, slot=None, pos=None) == wg.WG_OK
    assert lib_read(rows=0) == wg.WG_OK and lib_read(k=None, v=None) == wg.WG_OK


def test_library_refuses_scratch_and_attention():
    h = C.c_void_p()
    for bad in ((0, 8, 2, 64), (4, 0, 2, 64), (4, 8, 0, 64), (4, 8, 3, 64), (4, 1, 2, 64), (4, 8, 2, 24), (4, 8, 2, 272), (4, 8, 2, 0), (4, 70000, 2, 64),
                (4, 2048, 1025, 64)):
        assert lib.wg_attend_create(*bad, C.byref(h)) == wg.WG_ERR_ARG and not h.value
    assert lib.wg_attend_create(4, 8, 2, 64, None) == wg.WG_ERR_ARG
    lib.wg_attend_free(None)
    c = struct()
    assert lib.wg_kv_attend(None, C.addressof(c), 0x1000, 512, 0x1000, 512, None, 0, 8, 0x1000, 5, 5, 0x1000, 4, None, None, None, 4, 1.0, 0, 1,
                            None) == wg.WG_ERR_ARG


# ---- frequencies -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("how", [dict(), dict(base=500000.0), dict(factor=4.0), dict(factor=8.0, original=8192, low=1.0, high=4.0),
                                 dict(factor=0.5, original=100.0, low=0.0, high=32.0), dict(original=8192.0, low=1.0, high=4.0)])
@pytest.mark.parametrize("rot", [2, 16, 64, 128, 256])
def test_frequencies(how, rot):
    got = np.zeros(rot // 2)
    full = dict(dict(base=10000.0, factor=1.0, original=0.0, low=0.0, high=0.0), **how)
    assert lib.wg_rope_frequencies(rot, *(float(full[k]) for k in ("base", "factor", "original", "low", "high")), got.ctypes.data_as(C.c_void_p)) == 0
    assert got.tolist() == pytest.approx(ref.frequencies(rot, **full), rel=1e-14)


def test_frequencies_refused():
    out = np.zeros(200).ctypes.data_as(C.c_void_p)
    nan, inf = float("nan"), float("inf")
    for bad in ((0, 1e4, 1, 0, 0, 0), (15, 1e4, 1, 0, 0, 0), (-2, 1e4, 1, 0, 0, 0), (258, 1e4, 1, 0, 0, 0), (16, 0, 1, 0, 0, 0), (16, nan, 1, 0, 0, 0),
                (16, inf, 1, 0, 0, 0), (16, 1e4, 0, 0, 0, 0), (16, 1e4, inf, 0, 0, 0), (16, 1e4, nan, 0, 0, 0), (16, 1e4, 2, -1, 0, 0),
                (16, 1e4, 2, nan, 0, 0), (16, 1e4, 2, 100, 4, 4), (16, 1e4, 2, 100, -1, 4), (16, 1e4, 2, 100, 1, inf), (16, 1e4, 2, 100, nan, 4)):
        assert lib.wg_rope_frequencies(*bad, out) == wg.WG_ERR_ARG
    assert lib.wg_rope_frequencies(16, 1e4, 1, 0, 0, 0, None) == wg.WG_ERR_ARG
    for bad in ((None, 8, 4, 1.0, 0x1000), (out, 0, 4, 1.0, 0x1000), (out, 129, 4, 1.0, 0x1000), (out, 8, 0, 1.0, 0x1000), (out, 8, 4, 1.0, None)):
        assert lib.wg_rope_table(*bad, None) == wg.WG_ERR_ARG


@pytest.mark.parametrize("how", [dict(rot_dim=8), dict(rot_dim=24), dict(rot_dim=0), dict(rot_dim=272), dict(n_pos=0)])
def test_a_rope_refuses(no_library, how):  # noqa: F811
    with pytest.raises(ValueError):
        binding.Rope(**dict(dict(n_pos=10, rot_dim=32), **how))


# ---- the plain forms on cases made by hand ------------------------------------------------------------------------
def test_plain_rotation_by_hand():
    x = torch.tensor([[[1.0, 0.0, 0.0, 2.0, 5.0]]])
    quarter = [np.pi / 2, np.pi / 2]
    assert torch.allclose(ref.rotate(x, torch.tensor([1]), quarter, False), torch.tensor([[[0.0, -2.0, 1.0, 0.0, 5.0]]], dtype=torch.float64), atol=1e-15)
    assert torch.allclose(ref.rotate(x, torch.tensor([1]), quarter, True), torch.tensor([[[0.0, 1.0, -2.0, 0.0, 5.0]]], dtype=torch.float64), atol=1e-15)


def test_plain_codes_by_hand():
    codes, scale = ref.codes_of(torch.tensor([[127.0, -63.5, 0.4, 0.5, 1.5], [0.0, 0.0, 0.0, 0.0, 0.0], [1.0, float("nan"), 2.0, 3.0, 4.0]]), torch.int8)
    assert codes[:2].tolist() == [[127, -64, 0, 0, 2], [0] * 5] and scale[:2].tolist() == [1.0, 1.0] and scale[2].isnan()
    codes, scale = ref.codes_of(torch.tensor([[896.0, -17.0, 2.0 ** -8, 1.0]]), E4M3)
    assert codes.float().tolist() == [[448.0, -8.0, 2.0 ** -9, 0.5]] and scale.tolist() == [2.0]


def test_plain_attention_by_hand():
    """Two positions of one head with weights 1/4 and 3/4; a block that is not there; a window of one."""
    k = torch.zeros((3, 2, 1, 16), dtype=torch.float64)
    v = torch.zeros((3, 2, 1, 16), dtype=torch.float64)
    k[2, 0, 0, 0], k[2, 1, 0, 0] = 0.0, np.log(3.0)
    v[2, 0, 0, 1], v[2, 1, 0, 1] = 4.0, 8.0
    q = torch.zeros((1, 1, 16))
    q[0, 0, 0] = 2.0
    table = torch.tensor([[2, -1]])
    for pos, window, want, lse in ((1, 0, 7.0, np.log(4.0)), (1, 1, 8.0, np.log(3.0)), (3, 0, 7.0, np.log(4.0)), (0, 0, 4.0, 0.0)):
        out, got, _, _ = ref.attend(q, k, v, table, [0], [pos], 0.5, window)
        assert out[0, 0, 1].item() == pytest.approx(want) and got.item() == pytest.approx(lse)
    out, got, _, _ = ref.attend(q, k, v, table, [0], [3], 0.5, 2)
    assert (out == 0).all() and got.item() == -np.inf
