"""Windowed chunks of very many items, and of few rows beside a scratch area that they do not need."""
import pytest
import torch

import serving_reference as ref
from test_gpu_window import Paged, check, check_chunk, chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 64), (32, 8, 128)])
def test_chunk_items_of_many_rounds(hq, hkv, d):
    """More than 32 items for every CTA of one launch: a lane then works out a second item."""
    lens = [20 + (b * 53) % 150 for b in range(640)]
    rows = [n - (b % 7) * (n > 60) for b, n in enumerate(lens)]
    per_item = 2 * (128 // (hq // hkv))
    items = sum(-(-m // per_item) for m in rows) * hkv
    assert items > 32 * torch.cuda.get_device_properties(0).multi_processor_count
    p = Paged(lens, hkv, d, seed=71)
    q = p.rows(sum(rows), hq)
    p.forget([n - m for n, m in zip(lens, rows)], 50, 3)
    check_chunk(p, q, rows, chunk(p, q, rows, 50, 3), 50, 3)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 64)])
@pytest.mark.parametrize("rows", [[1, 1, 1, 0], [3, 1, 5, 2]])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 20), (5000, 0)])
def test_few_rows_on_fp8_pages_beside_a_scratch_area(window, sinks, rows, hq, hkv, d):
    """One by one from the codes: one launch, the scratch area not written, the FP8 kernels' tolerance.  (Eighty rows and kv heads over
    2064 tokens at head_dim 128 are no longer few: they go through the area, K and V off by 2^-8 of themselves there, which moves a
    score by 2^-8 of the row's reach, and a weight and the weights' sum by as much.)"""
    lens = [900, 17, 2049, 65]
    p = Paged(lens, hkv, d, fp8=True, seed=72)
    scratch = torch.full((p.cache.skv_prefill_scratch_bytes(),), 0x5A, dtype=torch.uint8, device="cuda")
    p.cache.skv_set_prefill_scratch(scratch)
    q = p.rows(sum(rows), hq)
    p.forget([n - m for n, m in zip(lens, rows)], window, sinks)
    few = len(lens) * max(rows) * hkv * min(window + sinks, 16 * p.table.shape[1]) * d <= 19200000
    assert few or (max(rows), hkv, d, window) == (5, 4, 128, 5000)
    before = p.cache.skv_launch_count()
    out = chunk(p, q, rows, window, sinks)
    assert p.cache.skv_launch_count() == before + (1 if few else 2)
    if few:
        check_chunk(p, q, rows, out, window, sinks)
        assert bool((scratch == 0x5A).all())
    else:
        at = 0
        for b, (n, m) in enumerate(zip(lens, rows)):
            want, size, reach = ref.attention(q[at:at + m], p.k[b], p.v[b], torch.arange(n - m, n), window, sinks)
            tol = ref.attention_tolerance(want, size, reach, n, False) + size * (2 ** -8 + 2 * 2 ** -8 * reach)
            assert bool(((out[at:at + m].double().cpu() - want).abs() <= tol).all())
            at += m
    assert p.cache.skv_get_status() == 0
    p.cache.skv_set_prefill_scratch(None)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rows,left", [([1, 1, 1, 1], 1), ([70, 33, 100, 64], 3)])
def test_rows_of_requests_that_were_refused(rows, left, fp8):
    """A step's table with requests that add no row (refused ones) beside others, their pages and lengths whatever they were."""
    lens = [900, 33, 2049, 65]
    p = Paged(lens, 2, 128, fp8, seed=73)
    kept = [m if b != left else 0 for b, m in enumerate(rows)]
    q = p.rows(sum(kept), 8)
    p.table_dev = p.table_dev.clone()
    p.table_dev[left] = -1
    out = chunk(p, q, kept, 100, 4)
    at = 0
    for b, (n, m) in enumerate(zip(lens, kept)):
        want = ref.attention(q[at:at + m], p.k[b], p.v[b], torch.arange(n - m, n), 100, 4)
        check(out[at:at + m], want + (n, fp8, float(p.v[b].double().abs().max())), f"sequence {b}")
        at += m
    assert p.cache.skv_get_status() == 0
