"""Attention on FP8 pages of queries next to nothing: scores that are next to nothing, so the mean of V."""
import random

import pytest
import torch

import pages_reference as pages
import serving_reference as ref
from test_gpu_pages import check_rows, chunk_runs, i32, some_lists
from test_gpu_window import Paged

pytestmark = pytest.mark.gpu

TINY_ROWS = [-120, -125, -126, -127, -128, -129, -130, -132, -133]


def tiny_queries(rows, hq, d, g):
    """Rows whose largest element is 2^-120 down to the smallest that bf16 has, and some of zeros."""
    q = torch.randint(-1, 2, (rows, hq, d), generator=g).double()
    q[..., 3] = 1.0
    for i in range(rows):
        for h in range(hq):
            q[i, h] *= 2.0 ** TINY_ROWS[(i * hq + h) % len(TINY_ROWS)]
    q[rows // 2, 0] = 0.0
    assert q.abs().max() < 2.0 ** -100
    got = q.to(torch.bfloat16)
    assert torch.equal(got.double(), q)                       # (powers of two: subnormal ones are there as they are)
    return got


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64), (4, 4, 128)])
def test_fp8_decode_of_queries_next_to_nothing(hq, hkv, d):
    """Scores that are next to nothing: the mean of V, on lists and in full."""
    p = Paged([500] * 9, hkv, d, True, seed=d)
    q = tiny_queries(9, hq, d, p.g)
    lists, counts = some_lists(random.Random(d), [32] * 9, hkv, 20)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(b, b, [499]) for b in range(9)])
    whole = torch.arange(32, dtype=torch.int32).expand(9, hkv, 32)
    full = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(9, hq), dtype=torch.uint8, device="cuda")
    p.cache.skv_decode_attn_window(0, q.cuda(), p.table_dev, p.lens_dev, full, ws, 10000, 0)
    check_rows(p, q, full, whole, torch.full((9, hkv), 32), [(b, b, [499]) for b in range(9)])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("hq,hkv,d,run", [(8, 2, 128, 16), (6, 2, 64, 5)])
def test_fp8_chunks_of_queries_next_to_nothing(hq, hkv, d, run, variant):
    n, a = 400, 2 * run
    p = Paged([n], hkv, d, True, seed=d)
    p.cache.skv_set_prefill_variant(variant)
    q = tiny_queries(a, hq, d, p.g)
    runs = chunk_runs([n], [a], a, run)
    lists, counts = some_lists(random.Random(run), [n // 16] * 2, hkv, 20)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, a, run=run)
    check_rows(p, q, out, lists, counts, runs)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("scratch", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_fp8_prefill_of_queries_next_to_nothing(hq, hkv, d, scratch):
    """Every page, and every page that a window reaches.  With a scratch area the values are rounded to bf16 there (2^-8 of each: 2^-8 sum w |v|) and
    the probabilities are bf16; keys are as well, which scores next to nothing do not hear."""
    n, a = 400, 40
    p = Paged([n], hkv, d, True, seed=d)
    if scratch:
        p.cache.skv_set_prefill_scratch(torch.empty(p.cache.skv_prefill_scratch_bytes(), dtype=torch.uint8, device="cuda"))
    q = tiny_queries(a, hq, d, p.g)
    pos, group = torch.arange(n - a, n), hq // hkv
    for window in (None, 100000):
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        if window is None:
            p.cache.skv_prefill_attn(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, out, a)
        else:
            p.cache.skv_prefill_attn_window(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, out, a, window)
        for h in range(hkv):
            mine = slice(None), slice(h * group, (h + 1) * group)
            want = pages.attention(q[mine], p.k[0][:, h], p.v[0][:, h], pos, list(range(n // 16)))
            tol = ref.attention_tolerance(*want, n, not scratch, float(p.v[0].abs().max())) + (want[1] * 2 ** -8 if scratch else 0.0)
            assert bool(((out[mine].double().cpu() - want[0]).abs() <= tol).all()), (window, h)
    assert p.cache.skv_get_status() == 0
