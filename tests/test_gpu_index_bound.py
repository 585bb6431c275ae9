"""skv_index_pages without row offsets: one new token per sequence, and the bound on new tokens is not read."""
import pytest

from paper_2604_22782_b200 import binding as B
from test_gpu_pages import check_index, i32, index_of
from test_gpu_window import Paged

pytestmark = pytest.mark.gpu


def test_index_of_a_step_does_not_read_the_bound():
    """Without offsets there is one new token per sequence, whatever the bound says."""
    lens = [16, 33, 48, 0]
    p = Paged(lens, 2, 64, seed=3)
    _, [(codes, scales)] = index_of(p.cache)
    for bound in (0, -5):
        codes.zero_(), scales.zero_()
        p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, max_q_len=bound)
        check_index(p, codes, scales, [max(n - 1, 0) // 16 for n in lens], [n // 16 for n in lens])
        with pytest.raises(B.SkvError):
            p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, i32([0, 1, 2, 3, 3]), bound)
    assert p.cache.skv_get_status() == 0
