"""What the host code of a paged cache's contents launches and refuses, without a GPU: over stand-ins for the CUDA runtime."""
import pytest

from test_launches_host import fake, lines  # noqa: F401

HEAD = """
    class Cache(C.Structure):
        _fields_ = [(n, C.c_void_p) for n in ("k", "v", "ks", "vs")] + [(n, C.c_int) for n in ("storage", "n_blocks", "block_size", "n_heads", "head_dim")]
    class Rope(C.Structure):
        _fields_ = [("table", C.c_void_p)] + [(n, C.c_int) for n in ("n_pos", "rot", "inter")]
    P, I, L = C.c_void_p, C.c_int, C.c_int64
    lib.wg_kv_attend.argtypes = [P, P, P, L, P, L, P, I, I, P, L, I, P, I, P, P, P, I, C.c_float, I, I, P]
    lib.wg_kv_write.argtypes = [P, P, L, P, L, P, L, P, L, I, I, P, P, P, I, P, P]
    lib.wg_kv_read.argtypes = [P, P, L, I, P, I, P, P, P, I, I, P]
    lib.wg_rope_table.argtypes = [P, I, I, C.c_double, P, P]
    def cache(storage=0, H=8, D=128, n_blocks=1000, block=16):
        s = at if storage > 1 else None
        return Cache(at, at, s, s, storage, n_blocks, block, H, D)
    scratch = C.c_void_p()
    def attend(c, n=4, Hq=32, dtype=0, q=at, qs=None, out=at, os=None, lse=None, table=at, stride=64, cols=64, len=at, n_seq=64, seq=None, pos=None, slot=None,
               window=0, group=1, handle=None, scale=1.0):
        w = Hq * c.head_dim
        return lib.wg_kv_attend(handle or scratch, C.byref(c), q, qs or w, out, os or w, lse, dtype, Hq, table, stride, cols, len, n_seq, seq, pos, slot, n, scale,
                                window, group, None)
    def launches():
        return sum(x.startswith("launch") for x in log())
"""


@pytest.mark.parametrize("storage", [0, 1, 2, 3])
def test_launches_of_an_attention(fake, storage):  # noqa: F811
    """One kernel and the one that joins; with groups a plan in front; batches beyond what one launch takes one after the other."""
    got = lines(fake, HEAD + f"""
    c, dtype = cache({storage}), {2 if storage == 1 else 0}
    assert lib.wg_attend_create(3000, 32, 8, 128, C.byref(scratch)) == 0
    for how in (dict(), dict(n=64), dict(group=4), dict(n=2000, n_seq=2000), dict(n=2000, n_seq=2000, group=5), dict(n=0), dict(window=7)):
        fake.fake_reset(-1)
        print(attend(c, dtype=dtype, **how), launches())
    for fails in range(2):
        fake.fake_reset(fails)
        print(attend(c, dtype=dtype), lib.wg_last_cuda_error())
        fake.fake_reset(-1)
        print(attend(c, dtype=dtype), launches())
    """)
    assert got == ["0 2", "0 2", "0 3", "0 12", "0 18", "0 0", "0 2"] + ["-5 701", "0 2"] * 2


def test_attention_refuses(fake):  # noqa: F811
    """Nothing is launched for a call that is refused."""
    got = lines(fake, HEAD + """
    assert lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)) == 0
    fake.fake_reset(-1)
    odd = at + 8
    bad = [dict(n=-1), dict(n=51), dict(dtype=1), dict(dtype=2), dict(dtype=3), dict(Hq=16), dict(Hq=64), dict(q=None), dict(out=None), dict(q=odd), dict(out=odd),
           dict(qs=4095), dict(qs=4092), dict(os=4100), dict(table=None), dict(cols=0), dict(stride=63), dict(n_seq=0), dict(len=None), dict(n=5, n_seq=4),
           dict(seq=at), dict(pos=at), dict(slot=at), dict(seq=at, pos=at), dict(seq=at, slot=at), dict(window=-1), dict(group=0), dict(group=33),
           dict(scale=float('nan')), dict(scale=float('inf')), dict(scale=3e38)]
    for how in bad:
        assert attend(cache(), **how) == -1, how
    for c in (cache(H=4), cache(D=64), cache(1), cache(n_blocks=1 << 28, block=16), cache(n_blocks=0), cache(4)):
        assert attend(c) == -1
    print(launches(), attend(cache()), attend(cache(), seq=at, pos=at, slot=at, len=None, n_seq=1), attend(cache(n_blocks=(1 << 28) - 1)), launches())
    """)
    assert got == ["0 0 0 0 6"]


@pytest.mark.parametrize("allocation", range(6))
def test_no_room_for_scratch(fake, allocation):  # noqa: F811
    got = lines(fake, HEAD + f"""
    fake.fake_no_room({allocation})
    print(lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)), scratch.value, lib.wg_last_cuda_error())
    fake.fake_no_room(-1)
    print(lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)), attend(cache()))
    lib.wg_attend_free(scratch)
    """)
    assert got == ["-5 None 2", "0 0"]


@pytest.mark.parametrize("T,Hq,H,D", [(1, 32, 8, 128), (12001, 32, 8, 128), (100, 0, 1, 16), (300000, 64, 64, 256), (7, 65535, 1024, 64)])
def test_launches_of_a_write(fake, T, Hq, H, D):  # noqa: F811
    """One kernel: lane groups enough for every vector of every token."""
    got = lines(fake, HEAD + f"""
    c, r = cache(2, {H}, {D}, 1 << 20), Rope(at, 100, 16, 0)
    fake.fake_reset(-1)
    print(lib.wg_kv_write(C.byref(c), at, {H * D}, at, {H * D}, at if {Hq} else None, {Hq * D}, at if {Hq} else None, {Hq * D}, {Hq}, 0, C.byref(r), at, at, {T}, None, None))
    print(*log())
    """)
    assert got[0] == "0" and got[1].count("launch") == 1
    x, y, z = (int(n) for n in got[1].split()[1:])
    lanes = 4 if D <= 64 else 8 if D <= 128 else 16
    assert x * 256 >= T * lanes > (x - 1) * 256 and 2 + (Hq > 0) <= y <= 65535 and z == 1
    assert any(y == -(-Hq // per) + 2 * -(-H // per) for per in range(1, 9))


@pytest.mark.parametrize("rows", [1, 700, 300000, 2 ** 31 - 1])
def test_launches_of_a_read(fake, rows):  # noqa: F811
    got = lines(fake, HEAD + f"""
    c = cache(3)
    fake.fake_reset(-1)
    print(lib.wg_kv_read(C.byref(c), at, 8, 8, at, 4, at, at, None, 0, {rows}, None))
    print(*log())
    fake.fake_reset(0)
    print(lib.wg_kv_read(C.byref(c), at, 8, 8, at, 4, at, at, None, 0, {rows}, None))
    """)
    assert got[0] == "0" and got[2] == "-5"
    x, y, z = (int(n) for n in got[1].split()[1:])
    assert any(x == -(-rows // per) for per in range(2, 33)) and (y, z) == (2, 1)


def test_launches_of_a_table_of_angles(fake):  # noqa: F811
    got = lines(fake, HEAD + """
    freq = (C.c_double * 64)(*[1.0] * 64)
    fake.fake_reset(-1)
    print(lib.wg_rope_table(freq, 64, 100, 1.0, at, None), lib.wg_rope_table(freq, 64, 2 ** 31 - 1, 1.0, at, None))
    print(*log(), sep=' | ')
    """)
    assert got == ["0 0", "launch 25 1 1 | launch 9472 1 1"]
