"""What the kernels' launches ask for, by arithmetic; no device."""
import ctypes

import pytest


def hooks():
    from paper_2604_22782_b200 import build
    return ctypes.CDLL(build.build_test_hooks())


@pytest.mark.parametrize("window,most", [(0, 239), (1, 447)])
def test_three_ctas_of_the_fp8_decode_kernel_fit_an_sm(window, most):
    """An SM has 228 KB, a CTA takes 1 KB beside its own: three of them have 76800 bytes each.  Rings, operands and barriers are
    74832 bytes, with a window 64 more for its token sets; what is left, in pieces of 128, holds the tables: 8 B + 4 bytes,
    with a window 4 B + 4 (a length and a page count per sequence, the counts alone).  1920 bytes: 239; 1792: 447."""
    f = hooks().skv_test_fp8_decode_smem_bytes
    f.restype = ctypes.c_size_t
    room = 228 * 1024 // 3 - 1024
    assert f(128, most, window) <= room < f(128, most + 1, window)
