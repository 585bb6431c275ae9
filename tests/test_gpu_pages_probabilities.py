"""Decode over listed bf16 pages, and chunks a row at a time: probabilities are held as two bf16 terms, so that their rounding is far
below the result's."""
import math
import random

import pytest
import torch

import pages_reference as pages
from test_gpu_pages import chunk_runs, i32, some_lists
from test_gpu_window import Paged

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 128), (8, 1, 128), (6, 2, 64), (16, 2, 64), (4, 4, 128)]


def check_fine(p, q, out, lists, counts, rows_of):
    """serving_reference's bound for bf16 pages with 2^-16 (2^-8 of what a first bf16 term leaves, which is 2^-8 of it at most) in the place of 2^-8
    for a probability: the result to bf16 2^-8, scores 2 x 128 additions off by 2^-23 of the products each, exp2 and the sums 2^-15."""
    hkv = lists.shape[1]
    group = q.shape[1] // hkv
    for i, (b, row, pos) in enumerate(rows_of):
        for h in range(hkv):
            mine = slice(row, row + len(pos)), slice(h * group, (h + 1) * group)
            want, size, reach = pages.attention(q[mine], p.k[b][:, h], p.v[b][:, h], torch.tensor(pos), lists[i, h, :counts[i, h]].tolist())
            tol = want.abs() * 2 ** -8 + size * (2 ** -16 + 2 * 128 * 2 ** -23 * reach + 2 ** -15)
            err = (out[mine].double().cpu() - want).abs()
            assert bool((err <= tol).all()), f"list {i} head {h}: {(err / tol.clamp(min=1e-30)).max().item():.2f} of what rounding allows"


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("width", [1, 9, 60])
def test_decode_where_values_cancel(hq, hkv, d, width):
    """V of either sign: the result is small beside what is summed."""
    lens = [17, 100, 257, 1000]
    p = Paged(lens, hkv, d, seed=width)
    q = p.rows(len(lens), hq)
    lists, counts = some_lists(random.Random(width), [-(-n // 16) for n in lens], hkv, width)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_fine(p, q, out, lists, counts, [(b, b, [n - 1]) for b, n in enumerate(lens)])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_rows_of_chunks_where_values_cancel(hq, hkv, d):
    lens, new = [40, 300, 1201], [9, 1, 20]
    p = Paged(lens, hkv, d, seed=hq)
    p.cache.skv_set_prefill_variant(1)
    q = p.rows(sum(new), hq)
    runs = chunk_runs(lens, new, 20, 4)
    lists, counts = some_lists(random.Random(d), [(r[2][-1] // 16 + 1 if r[2] else 0) for r in runs], hkv, 30)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, 9, 10, 30]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, 20, run=4)
    check_fine(p, q, out, lists, counts, runs)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_infinite_values_are_what_they_are(hq, hkv, d):
    """An infinite V of some weight gives infinity in its dim, two of unlike sign NaN, and nothing elsewhere."""
    n = 64
    p = Paged([n], hkv, d, seed=3)
    v = p.v[0].clone()
    v[3, 0, 5], v[20, 0, 9], v[21, hkv - 1, 11], v[50, hkv - 1, 11] = math.inf, -math.inf, math.inf, -math.inf
    slots = (p.table[0].long()[torch.arange(n) // 16] * 16 + torch.arange(n) % 16).cuda()
    p.cache.skv_append(0, p.k[0].cuda(), v.cuda(), slots)
    q = p.rows(1, hq)
    q[0, 0] = 0.0                                             # (equal weights: powers of two, whose second term is 0)
    lists, counts = torch.arange(4, dtype=torch.int32).expand(1, hkv, 4).contiguous(), torch.full((1, hkv), 4, dtype=torch.int32)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    got = out[0].float().cpu().view(hkv, hq // hkv, d)
    assert bool((got[0, :, 5] == math.inf).all()) and bool((got[0, :, 9] == -math.inf).all()) and bool(got[hkv - 1, :, 11].isnan().all())
    got[0, :, 5] = got[0, :, 9] = got[hkv - 1, :, 11] = 0.0
    assert bool(got.isfinite().all()) and p.cache.skv_get_status() == 0
