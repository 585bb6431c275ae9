"""NaN and infinities in queries and in tokens that are seen: the definition's result is then NaN, and no other row's, head's
or sequence's result is touched."""
import pytest
import torch

import serving_reference as ref
from test_gpu_window import Paged, chunk, decode

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
SHAPES = [(8, 2, 128), (4, 4, 128), (8, 1, 128), (6, 2, 64), (4, 4, 64)]


def spoil_keys(p, b, tokens):
    """The keys of some tokens of sequence b become NaN; their values stay (on FP8 pages: are stored anew)."""
    bad = torch.full((len(tokens),) + p.k[b].shape[1:], NAN, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_append(0, bad, p.v[b][tokens].bfloat16().cuda(), ref.slots_of(p.table, b, tokens).cuda())
    p.k[b][tokens] = NAN


def compare(got, want, n, fp8, v_max):
    out, size, reach = want
    got = got.double().cpu()
    assert torch.equal(got.isnan(), out.isnan())
    tol = ref.attention_tolerance(out, size, reach, n, fp8, v_max)
    assert bool((out.isnan() | ((got - out).abs() <= tol)).all())


def compare_decode(p, q, out, window, sinks):
    for b, n in enumerate(p.lens):
        want = ref.attention(q[b:b + 1], p.k[b], p.v[b], torch.tensor([n - 1]), window, sinks)
        compare(out[b:b + 1], want, min(n, window + sinks), p.fp8, float(p.v[b].double().abs().max()) if n else 0.0)


def compare_chunk(p, q, rows, out, window, sinks):
    at = 0
    for b, (n, m) in enumerate(zip(p.lens, rows)):
        want = ref.attention(q[at:at + m], p.k[b], p.v[b], torch.arange(n - m, n), window, sinks)
        compare(out[at:at + m], want, n, p.fp8, float(p.v[b].double().abs().max()) if n else 0.0)
        at += m


# one sequence shared by a cluster, a page a warp; a few; a CTA for each; short ones without and with one token
LENGTHS = [[1040], [1040, 33, 600, 17, 0, 1, 2049], [300 + b for b in range(160)]]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("lens", LENGTHS)
def test_window_decode_of_a_query_that_is_not_finite(lens, hq, hkv, d, fp8):
    p = Paged(lens, hkv, d, fp8, seed=51)
    q = p.rows(len(lens), hq)
    q[0, 1] = NAN                                         # a whole head
    if len(lens) > 1:
        q[1, hq - 1, 3] = NAN                             # an element
        q[2, 0, 5] = INF
    for window, sinks in ((1024, 0), (20, 3)):
        compare_decode(p, q, decode(p, q, window, sinks), window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("lens", LENGTHS)
@pytest.mark.parametrize("first,count", [(272, 16), (100, 1), (64, 200), (0, 300)])
def test_window_decode_of_keys_that_are_not_finite(lens, hq, hkv, d, first, count, fp8):
    """A page, a token, several pages, and (of longer sequences) everything up to the window's last tokens."""
    p = Paged(lens, hkv, d, fp8, seed=52)
    spoil_keys(p, 0, torch.arange(first, first + count))
    q = p.rows(len(lens), hq)
    for window, sinks in ((1024, 0), (1024, 4), (3, 2), (7, 0)):
        compare_decode(p, q, decode(p, q, window, sinks), window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("variant", [0, 1])
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 1, 5], [40, 33, 70]])
def test_window_chunk_of_what_is_not_finite(rows, variant, hq, hkv, d, fp8):
    """Few rows, which go one by one unless a kernel is asked for, and more of them: one answer."""
    lens = [1040, 33, 700]
    p = Paged(lens, hkv, d, fp8, seed=53)
    p.cache.skv_set_prefill_variant(variant)
    spoil_keys(p, 2, torch.arange(688, 700) if variant else torch.arange(640, 656))
    q = p.rows(sum(rows), hq)
    q[0, 1] = NAN
    q[rows[0], 0, 7] = INF
    for window, sinks in ((1024, 0), (30, 4)):
        compare_chunk(p, q, rows, chunk(p, q, rows, window, sinks), window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64), (5, 1, 128)])
@pytest.mark.parametrize("first,count", [(1184, 384), (1500, 900), (2800, 216), (64, 1)])
@pytest.mark.parametrize("sequences", [1, 3])
def test_chunk_shared_by_a_cluster_of_what_is_not_finite(sequences, first, count, hq, hkv, d):
    """All the keys of one CTA's part are NaN and no others (one sequence, window 2900: blocks 17 to 22 of the 46 from token 96
    on), of several, those behind the first row's place, a single one; and a NaN query."""
    lens, rows = [3020, 2500, 3000][:sequences], [17, 20, 5][:sequences]
    p = Paged(lens, hkv, d, seed=54)
    p.cache.skv_set_prefill_variant(2)
    spoil_keys(p, 0, torch.arange(first, first + count))
    q = p.rows(sum(rows), hq)
    q[2, 1] = NAN
    q[4, 0, 9] = INF
    for window, sinks in ((2900, 0), (1600, 100), (1200, 0), (210, 3)):
        compare_chunk(p, q, rows, chunk(p, q, rows, window, sinks), window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("worker,merge", [(1, 0), (2, 1), (2, 2)])
@pytest.mark.parametrize("lens", LENGTHS)
def test_plain_decode_of_what_is_not_finite(lens, worker, merge, hq, hkv, d, fp8):
    """The call without a window: a warp per range, a CTA per range, with the merge launch and without."""
    p = Paged(lens, hkv, d, fp8, seed=55)
    p.cache.skv_set_decode_worker(worker)
    p.cache.skv_set_decode_merge(merge)
    spoil_keys(p, 0, torch.arange(272, 288))
    q = p.rows(len(lens), hq)
    if len(lens) > 1:
        q[1, 1] = NAN
        q[2, 0, 5] = NAN
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(len(lens), hq), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn(1, q.cuda(), p.table_dev, p.lens_dev, out, ws)
    torch.cuda.synchronize()
    compare_decode(p, q, out, 1 << 30, 0)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8), (64, 8)])
@pytest.mark.parametrize("window", [0, 300])
def test_decode_of_many_fp8_sequences_with_a_query_that_is_not_finite(window, hq, hkv, value):
    """The tcgen05 kernel, without and with a window.  (An infinite element times a key's element is infinite or NaN for every
    token, so the definition's weights are NaN.)"""
    lens = [1 + (b * 37) % 600 for b in range(200)] + [1200]
    p = Paged(lens, hkv, 128, fp8=True, seed=56)
    q = p.rows(len(lens), hq)
    q[0, 0, 5] = value
    q[17, hq - 1, 127] = value
    q[200, 1] = value
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(len(lens), hq), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    if window:
        p.cache.skv_decode_attn_window(1, q.cuda(), p.table_dev, p.lens_dev, out, ws, window, 4)
    else:
        p.cache.skv_decode_attn(1, q.cuda(), p.table_dev, p.lens_dev, out, ws)
    torch.cuda.synchronize()
    compare_decode(p, q, out, window or 1 << 30, 4)
    assert p.cache.skv_get_status() == 0
