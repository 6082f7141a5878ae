"""Scratch of the attention that finds no memory, at each of its allocations, without a GPU."""
import pytest

from test_cache_host import HEAD
from test_launches_host import fake, lines  # noqa: F401


def test_how_many_allocations_there_are(fake):  # noqa: F811
    got = lines(fake, HEAD + """
    for allocation in range(9):
        fake.fake_no_room(allocation)
        print(lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)))
        fake.fake_no_room(-1)
        lib.wg_attend_free(scratch)
    """)
    assert got == ["-5"] * 7 + ["0"] * 2


@pytest.mark.parametrize("allocation", [0, 6])
def test_no_room_at_an_allocation(fake, allocation):  # noqa: F811
    got = lines(fake, HEAD + f"""
    fake.fake_no_room({allocation})
    print(lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)), scratch.value, lib.wg_last_cuda_error())
    fake.fake_no_room(-1)
    print(lib.wg_attend_create(50, 32, 8, 128, C.byref(scratch)), attend(cache()))
    lib.wg_attend_free(scratch)
    """)
    assert got == ["-5 None 2", "0 0"]
