"""What the host code launches, without a GPU: the library in a process of its own, over stand-ins for the CUDA runtime
(fake_cudart.c) that write the launches down."""
import os
import subprocess
import sys
import textwrap

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libfake_cudart.so")
    subprocess.check_call(["gcc", "-O1", "-std=c11", "-Wall", "-shared", "-fPIC", "-o", out, os.path.join(HERE, "fake_cudart.c")])
    return out


PRELUDE = """
import ctypes as C
fake = C.CDLL({fake!r}, mode=C.RTLD_GLOBAL)      # found before the runtime that the library is linked to
lib = C.CDLL({lib!r})
fake.fake_log.restype = C.c_char_p
lib.wg_beam_select.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p] + [C.c_int] * 5 + [C.c_void_p] * 4
lib.wg_kv_extend.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_void_p, C.c_void_p, C.c_int] + [C.c_void_p] * 4 + [C.c_int, C.c_void_p, C.c_void_p]
at = 1 << 20                                     # an address that nothing looks at
def log():
    return fake.fake_log().decode().split('\\n')[:-1]
"""


def lines(fake, body):
    code = PRELUDE.format(fake=fake, lib=os.path.join(ROOT, "paper_2507_16768_b200", "libwg.so")) + textwrap.dedent(body)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return r.stdout.splitlines()


@pytest.mark.parametrize("n_tokens,blocks", [(2049, 9), (2304, 9), (2305, 10), (2 ** 31 - 256, 2 ** 23 - 1), (2 ** 31 - 255, 2 ** 23), (2 ** 31 - 1, 2 ** 23)])
def test_extend_places_any_number_of_tokens(fake, n_tokens, blocks):
    got = lines(fake, f"""
        pool = C.c_void_p()
        assert lib.wg_kv_pool_create(100, 16, 4, C.byref(pool)) == 0
        fake.fake_reset(-1)
        print(lib.wg_kv_extend(pool, at, 8, 8, at, at, 4, at, at, at, at, {n_tokens}, None, None))
        print(*log(), sep='\\n')
    """)
    assert got == ["0", "launch 1 1 1", f"launch {blocks} 1 1"]


SELECT = """
    beam, n_req = C.c_void_p(), 400
    assert lib.wg_beam_create(30000, n_req, 8, 8, C.byref(beam)) == 0
    def select():
        return lib.wg_beam_select(beam, at, 0, 30000, None, 0, at, None, 0, n_req, 8, 8, 0, at, at, at, 77)
"""


def test_a_selection_that_was_cut_short_leaves_no_counts(fake):
    """The scan deals its items out from counters that the pick behind it sets back.  Where the pick could not be
    launched, they are set back all the same, behind the scan and on its stream."""
    got = lines(fake, SELECT + """
    fake.fake_reset(-1)
    print(select(), [l.split()[0] for l in log()])
    fake.fake_reset(1)
    print(select(), [l.split()[0] for l in log()], log()[-1])
    fake.fake_reset(-1)
    fake.fake_stale_error(0)
    print(select(), [l.split()[0] for l in log()], log()[-1])
    fake.fake_reset(-1)
    print(select(), [l.split()[0] for l in log()])
""")
    assert got == ["0 ['launch', 'launch']", "-5 ['launch', 'failed-launch', 'memset'] memset 0 512 on 77",
                   "-5 ['launch', 'memset'] memset 0 512 on 77", "0 ['launch', 'launch']"]


def test_new_scratch_is_ready_for_every_stream(fake):
    """What is set when a handle is made is queued on the default stream, which other streams do not wait for: the call
    ends when it is done."""
    got = lines(fake, """
        h = C.c_void_p()
        for make in (lambda: lib.wg_beam_create(30000, 4, 8, 8, C.byref(h)), lambda: lib.wg_kv_pool_create(100, 16, 4, C.byref(h))):
            fake.fake_reset(-1)
            print(make(), "memset on the default stream" in log(), log()[-1])
    """)
    assert got == ["0 True wait for the default stream"] * 2


@pytest.mark.parametrize("allocation", [0, 1, 2])
def test_a_failed_call_leaves_no_error_to_the_next(fake, allocation):
    """No memory for a handle: that call fails, and the next one, on another handle, does not."""
    got = lines(fake, SELECT + f"""
    other = C.c_void_p()
    fake.fake_reset(-1)
    fake.fake_no_room({allocation})
    print(lib.wg_beam_create(500, 4, 8, 8, C.byref(other)), other.value, lib.wg_last_cuda_error())
    print(select())
    fake.fake_no_room({allocation})
    print(lib.wg_kv_pool_create(100, 16, 4, C.byref(other)), other.value, lib.wg_last_cuda_error())
    print(lib.wg_kv_pool_create(100, 16, 4, C.byref(other)), select())
    fake.fake_reset(1)
    print(select(), lib.wg_last_cuda_error())
    fake.fake_reset(-1)
    print(select())
""")
    assert got == ["-5 None 2", "0", "-5 None 2", "0 0", "-5 701", "0"]
