"""Decode of few segments with a query head per kv head: of the CUDA cores' state of 128 dims an SM has one CTA of 8 warps, and the
clusters have to be there at once all the same."""
import random

import pytest
import torch

import serving_reference as ref
from test_gpu_pages import check_rows, some_lists
from test_gpu_window import Paged, check as check_window, decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [6, 7, 8, 9, 10])
@pytest.mark.parametrize("width", [64, 65, 128])
def test_few_segments_with_a_query_head_each(heads, width):
    p = Paged([3000], heads, 128, seed=heads)
    q = p.rows(1, heads)
    lists, counts = some_lists(random.Random(width), [188], heads, width)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(0, 0, [2999])])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("heads", [7, 8, 9])
def test_few_segments_with_a_query_head_each_over_a_window(heads):
    p = Paged([3000], heads, 128, seed=heads)
    q = p.rows(1, heads)
    got = decode(p, q, 2048, 4)
    want = ref.attention(q, p.k[0], p.v[0], torch.tensor([2999]), 2048, 4)
    check_window(got, want + (2048 + 4, False, 0.0), f"{heads} heads")
    assert p.cache.skv_get_status() == 0
