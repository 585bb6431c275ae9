"""Where skv_plan_release puts a row's pages on the stack, for totals beyond 32 bits, which no pool of a test's size reaches."""
import ctypes

import pytest


def place(before, have, room):
    """Of a warp that has seen `before` pages ahead of its own entries, the place of the one `have` (0 to 31) entries on; -1: no room."""
    from paper_2604_22782_b200 import build
    f = ctypes.CDLL(build.build_test_hooks()).skv_test_release_place
    f.argtypes, f.restype = [ctypes.c_int64, ctypes.c_int, ctypes.c_int], ctypes.c_int64
    return f(before, have, room)


@pytest.mark.parametrize("room", [0, 1, 5, 31, 32, 1000, 2 ** 31 - 40, 2 ** 31 - 1])
def test_places(room):
    for before in [0, 1, 4, 5, 31, 32, 999, 1000, 2 ** 31 - 64, 2 ** 31 - 33, 2 ** 31 - 32, 2 ** 31 - 2, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 5, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 7,
                   2 ** 40, room - 1, room, room + 1]:
        for have in (0, 1, 30, 31):
            want = max(before, 0) + have
            assert place(max(before, 0), have, room) == (want if want < room else -1), (before, have)
