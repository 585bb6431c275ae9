"""How decode attention over listed pages and over a window is cut, by arithmetic; no device."""
import ctypes

import pytest


def shape(listed, d, kernel, segments, pages, sm=148):
    from paper_2604_22782_b200 import build
    f = ctypes.CDLL(build.build_test_hooks()).skv_test_decode_shape
    f.argtypes = [ctypes.c_int] * 3 + [ctypes.c_int64] * 2 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    out = (ctypes.c_int * 4)()
    assert f(listed, d, kernel, segments, pages, sm, out) == 0
    return list(out)


@pytest.mark.parametrize("listed", [0, 1])
@pytest.mark.parametrize("kernel", [0, 1, 2])
@pytest.mark.parametrize("d", [64, 128])
def test_clusters_of_16_have_two_ctas_to_an_sm(listed, kernel, d):
    """A cluster's CTAs share a GPC, which may have fewer than 16 SMs: of 16 CTAs two have to fit an SM.  And clusters of 4-warp CTAs are all there
    at once, by what the kernel's launch bounds promise (over a window no bound says so)."""
    wide = 0
    for segments in list(range(1, 40)) + [64, 100, 148, 149, 300, 1000]:
        for pages in (1, 3, 4, 31, 32, 63, 64, 65, 128, 500, 4000):
            warps, stages, ranks, per_sm = shape(listed, d, kernel, segments, pages)
            assert warps in (4, 8) and stages in (1, 2) and ranks in (1, 2, 4, 8, 16)
            assert ranks <= 8 or per_sm >= 2, (segments, pages, warps, stages, ranks)
            assert not listed or warps == 8 or ranks == 1 or segments * ranks <= per_sm * 148, (segments, pages, warps, stages, ranks)
            wide += ranks > 8
    assert wide or kernel == 2                                # (clusters of 16 are there at all)
