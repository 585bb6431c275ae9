"""The kernels that windowed attention reaches only by a setting, a size or an alignment: each against the 64-bit statement."""
import pytest
import torch

import serving_reference as ref
from test_gpu_window import Paged, check, check_chunk, check_decode, chunk, decode

pytestmark = pytest.mark.gpu

LENS, ROWS = [900, 33, 128, 2049, 5, 300, 0, 17], [100, 33, 0, 513, 1, 17, 0, 2]


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 64), (8, 1, 64), (5, 1, 128)])
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 20), (300, 17), (129, 200), (5000, 0)])
def test_chunk_kernels_on_bf16_pages(hq, hkv, d, variant, window, sinks):
    p = Paged(LENS, hkv, d, seed=31)
    p.cache.skv_set_prefill_variant(variant)
    q = p.rows(sum(ROWS), hq)
    p.forget([n - m for n, m in zip(LENS, ROWS)], window, sinks)
    check_chunk(p, q, ROWS, chunk(p, q, ROWS, window, sinks), window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 20), (300, 17), (129, 200), (5000, 0)])
def test_chunk_on_fp8_pages_through_a_scratch_area(hq, hkv, d, window, sinks):
    """The code times its scale is rounded to bf16 there: K and V are off by 2^-8 of themselves, which moves a score by
    2^-8 of the row's reach (so every weight and their sum by as much) and the sum by 2^-8 sum w |v|."""
    p = Paged(LENS, hkv, d, fp8=True, seed=32)
    scratch = torch.full((p.cache.skv_prefill_scratch_bytes(),), 0xFF, dtype=torch.uint8, device="cuda")      # NaN as bf16
    p.cache.skv_set_prefill_scratch(scratch)
    q = p.rows(sum(ROWS), hq)
    p.forget([n - m for n, m in zip(LENS, ROWS)], window, sinks)
    for variant in (0, 2):
        p.cache.skv_set_prefill_variant(variant)
        before = p.cache.skv_launch_count()
        out = chunk(p, q, ROWS, window, sinks)
        assert p.cache.skv_launch_count() == before + 2
        row = 0
        for b, (n, m) in enumerate(zip(LENS, ROWS)):
            want, size, reach = ref.attention(q[row:row + m], p.k[b], p.v[b], torch.arange(n - m, n), window, sinks)
            tol = ref.attention_tolerance(want, size, reach, n, False) + size * (2 ** -8 + 2 * 2 ** -8 * reach)
            assert bool(((out[row:row + m].double().cpu() - want).abs() <= tol).all()), (variant, n, m)
            row += m
    assert p.cache.skv_get_status() == 0
    p.cache.skv_set_prefill_scratch(None)


def test_chunk_kernel_that_does_not_apply_is_refused():
    from paper_2604_22782_b200.binding import SKV_ERR_UNSUPPORTED, SkvError
    p = Paged([40], 2, 128, fp8=True, seed=33)
    p.cache.skv_set_prefill_variant(2)                                          # (no scratch area)
    with pytest.raises(SkvError) as e:
        chunk(p, p.rows(3, 4), [3], 8, 0)
    assert e.value.status == SKV_ERR_UNSUPPORTED


@pytest.mark.parametrize("fp8", [False, True])
def test_chunk_batches_beyond_one_launch(fp8):
    """More sequences than a launch holds, short and empty ones between, the last of them long."""
    lens = [b % 5 * 7 for b in range(2600)] + [400]
    rows = [min(n, b % 4) for b, n in enumerate(lens[:-1])] + [150]
    p = Paged(lens, 1, 64, fp8, seed=34, spare=1)
    q = p.rows(sum(rows), 2)
    check_chunk(p, q, rows, chunk(p, q, rows, 20, 3), 20, 3)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_chunk_rows_at_the_smallest_alignment(d):
    """Q and out 16 bytes (the tensor-memory kernel) and 4 bytes (the other one) off a 32-byte boundary."""
    p = Paged(LENS, 2, d, seed=35)
    n = sum(ROWS)
    q = p.rows(n, 6)
    cu = torch.tensor([0] + torch.tensor(ROWS).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    for off in (8, 2):
        room = [torch.zeros(n * 6 * d + 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        qd, out = (x[off:off + n * 6 * d].view(n, 6, d) for x in room)
        qd.copy_(q)
        room[1][:off] = 7.0
        room[1][off + n * 6 * d:] = 7.0
        p.cache.skv_prefill_attn_window(1, qd, cu, p.table_dev, p.lens_dev, out, max(ROWS), 100, 5)
        check_chunk(p, q, ROWS, out, 100, 5)
        assert bool((room[1][:off] == 7.0).all() and (room[1][off + n * 6 * d:] == 7.0).all())


def test_chunk_captured_and_replayed_with_other_inputs_and_on_two_streams():
    p = Paged(LENS, 2, 128, seed=36)
    qs = [p.rows(sum(ROWS), 8) for _ in range(2)]
    cu = torch.tensor([0] + torch.tensor(ROWS).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    qd = [q.cuda() for q in qs]
    outs = [torch.empty_like(x) for x in qd]
    streams, graphs = [torch.cuda.Stream() for _ in range(2)], []
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            p.cache.skv_prefill_attn_window(1, qd[i], cu, p.table_dev, p.lens_dev, outs[i], max(ROWS), 100, 5)
            streams[i].synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=streams[i]):
                p.cache.skv_prefill_attn_window(1, qd[i], cu, p.table_dev, p.lens_dev, outs[i], max(ROWS), 100, 5)
            graphs.append(g)
    for round_ in range(6):
        for i in range(2):
            qd[i].copy_(qs[(i + round_) % 2])
            outs[i].fill_(float("nan"))
        torch.cuda.synchronize()
        for _ in range(3):
            for i in range(2):
                with torch.cuda.stream(streams[i]):
                    graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            check_chunk(p, qs[(i + round_) % 2], ROWS, outs[i], 100, 5)


def test_chunk_of_large_scores():
    """Scores of some thousands, where a maximum that grows from block to block makes every earlier sum vanish."""
    lens, rows = [1200, 500], [700, 500]
    p = Paged(lens, 2, 128, seed=37, magnitude=20.0)
    ramp = torch.linspace(0.0, 1.0, 1200)[:, None, None]
    for b, n in enumerate(lens):
        p.k[b] = (p.k[b].abs().float() * ramp[:n]).bfloat16()
        slots = ref.slots_of(p.table, b, torch.arange(n)).cuda()
        p.cache.skv_append(0, p.k[b].cuda(), p.v[b].cuda(), slots)
    q = (p.rows(sum(rows), 8).abs().float() * 20).bfloat16()
    for window, sinks in ((600, 40), (100, 0)):
        check_chunk(p, q, rows, chunk(p, q, rows, window, sinks), window, sinks)


@pytest.mark.parametrize("variant,hq,hkv,d", [(1, 4, 4, 128), (2, 4, 4, 128), (2, 4, 4, 64), (1, 2, 2, 64), (2, 8, 2, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 20), (333, 70)])
def test_decode_arithmetic_by_setting(variant, hq, hkv, d, window, sinks):
    p = Paged(LENS, hkv, d, seed=38)
    p.cache.skv_set_decode_variant(variant)
    q = p.rows(len(LENS), hq)
    p.forget([n - 1 for n in LENS], window, sinks)
    check_decode(p, q, decode(p, q, window, sinks), window, sinks)


@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8), (64, 8), (24, 8)])
@pytest.mark.parametrize("window,sinks", [(300, 0), (350, 5), (257, 131), (1000, 4)])
@pytest.mark.parametrize("variant", [0, 2])
def test_decode_of_many_fp8_sequences(hq, hkv, window, sinks, variant):
    """Enough tiles for the tcgen05 kernel, by the table's width; lengths around tiles, pages and the window's ends."""
    edge = [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 300, 301, 383, 384, 385, 500, 1100]
    lens = [edge[b % len(edge)] + (b // len(edge)) % 3 * (edge[b % len(edge)] > 0) for b in range(190)] + [2900]
    p = Paged(lens, hkv, 128, fp8=True, seed=39)
    p.cache.skv_set_decode_variant(variant)
    q = p.rows(len(lens), hq)
    p.forget([n - 1 for n in lens], window, sinks)
    before = p.cache.skv_launch_count()
    out = decode(p, q, window, sinks)
    assert p.cache.skv_launch_count() - before == 1
    check_decode(p, q, out, window, sinks)
    assert bool((out[0] == 0).all()) and p.cache.skv_get_status() == 0


def test_decode_of_fp8_sequences_in_pieces():
    lens = [(11 * b) % 70 for b in range(9000)]
    p = Paged(lens, 1, 128, fp8=True, seed=40, spare=20)
    q = p.rows(len(lens), 4)
    before = p.cache.skv_launch_count()
    out = decode(p, q, 30, 2)
    assert p.cache.skv_launch_count() - before == 3
    for b in list(range(0, 20)) + list(range(4090, 4105)) + list(range(8185, 8200)) + [8999]:
        want = ref.attention(q[b:b + 1], p.k[b], p.v[b], torch.tensor([lens[b] - 1]), 30, 2)
        check(out[b:b + 1], want + (32, True, float(p.v[b].double().abs().max()) if lens[b] else 0.0), f"sequence {b}")
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("lens", [[32700, 9000], [0, 0], [16, 1], [32768, 1], [130, 32768], [5000, 0]])
@pytest.mark.parametrize("layer", [0, 1])
def test_decode_of_fp8_segments_shared_by_many_workers(lens, layer):
    """Few sequences whose table has room for enough tiles: a segment is joined from up to a worker per tile, whatever the
    workspace held before; layer 1 walks the other way."""
    p = Paged(lens, 8, 128, fp8=True, seed=41)
    width = torch.full((2, 2048), -1, dtype=torch.int32)
    width[:, :p.table.shape[1]] = p.table
    p.table = width
    p.table_dev = width.cuda()
    q = p.rows(2, 32)
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(2, 32), dtype=torch.uint8, device="cuda")
    outs = []
    for fill in (0, 0xFF, 0x5A):
        ws.fill_(fill)
        for _ in range(3):
            out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
            p.cache.skv_decode_attn_window(layer, q.cuda(), p.table_dev, p.lens_dev, out, ws, 32000, 700)
            outs.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(o, outs[0]) for o in outs)
    check_decode(p, q, outs[0], 32000, 700)
    assert p.cache.skv_get_status() == 0


def test_decode_of_fp8_sequences_captured_and_replayed():
    lens = [300 + 37 * b % 800 for b in range(200)]
    p = Paged(lens, 8, 128, fp8=True, seed=42)
    qs = [p.rows(len(lens), 16) for _ in range(2)]
    ws = torch.full((p.cache.skv_decode_workspace_bytes(len(lens), 16),), 0x77, dtype=torch.uint8, device="cuda")
    qd = qs[0].cuda()
    out = torch.empty_like(qd)
    s = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(s):
        for calls in (1, 2):
            p.cache.skv_decode_attn_window(1, qd, p.table_dev, p.lens_dev, out, ws, 600, 4)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                for _ in range(calls):
                    p.cache.skv_decode_attn_window(1, qd, p.table_dev, p.lens_dev, out, ws, 600, 4)
            graphs.append(g)
    for i in (0, 1, 0):
        qd.copy_(qs[i])
        for g in graphs:
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            for _ in range(3):
                g.replay()
            torch.cuda.synchronize()
            check_decode(p, qs[i], out, 600, 4)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64), (5, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("window,sinks", [(900, 0), (900, 40), (2000, 700), (1, 3000), (5000, 0), (2147483647, 2147483647)])
def test_chunk_of_few_rows_shared_by_a_cluster(hq, hkv, d, window, sinks):
    """Long windows and few rows: an item's key blocks are several CTAs', some of them with none or with keys that some rows do
    not see; what nobody sees is NaN."""
    lens, rows = [3000, 40, 1111, 5, 0, 2047], [17, 40, 1, 5, 0, 33]
    p = Paged(lens, hkv, d, seed=43)
    q = p.rows(sum(rows), hq)
    p.forget([n - m for n, m in zip(lens, rows)], window, sinks)
    out = chunk(p, q, rows, window, sinks)
    check_chunk(p, q, rows, out, window, sinks)
    assert torch.equal(out, chunk(p, q, rows, window, sinks))
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("sequences", [1, 2, 3, 4, 8])
def test_chunk_of_few_rows_captured_and_beside_another_stream(sequences):
    lens = [2500 + 100 * b for b in range(sequences)]
    rows = [20 + b for b in range(sequences)]
    p = Paged(lens, 4, 128, seed=44)
    q = p.rows(sum(rows), 16)
    cu = torch.tensor([0] + torch.tensor(rows).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    qd, outs = q.cuda(), [torch.empty(q.shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[0]):
        p.cache.skv_prefill_attn_window(1, qd, cu, p.table_dev, p.lens_dev, outs[0], max(rows), 2048, 4)
        streams[0].synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=streams[0]):
            p.cache.skv_prefill_attn_window(1, qd, cu, p.table_dev, p.lens_dev, outs[0], max(rows), 2048, 4)
    outs[0].fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            g.replay()
        p.cache.skv_prefill_attn_window(1, qd, cu, p.table_dev, p.lens_dev, outs[1], max(rows), 2048, 4, stream=streams[1])
    torch.cuda.synchronize()
    check_chunk(p, q, rows, outs[0], 2048, 4)
    assert torch.equal(outs[0], outs[1]) and p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 64), (4, 4, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 20), (700, 0), (129, 200), (5000, 0), (2147483647, 2147483647)])
@pytest.mark.parametrize("rows", [[1, 1, 0, 1, 1], [5, 17, 0, 1, 3], [12, 3, 2, 9, 5]])
def test_chunk_of_rows_that_go_one_by_one(hq, hkv, d, window, sinks, rows, fp8):
    """Through the decode kernel and, asked for, through the tile kernel: both against the definition, rows behind the last one left."""
    lens = [900, 17, 2, 2049, 65]
    p = Paged(lens, hkv, d, fp8, seed=45)
    q = p.rows(sum(rows), hq)
    p.forget([n - m for n, m in zip(lens, rows)], window, sinks)
    for variant in (0, 1):
        p.cache.skv_set_prefill_variant(variant)
        check_chunk(p, q, rows, chunk(p, q, rows, window, sinks), window, sinks)
        assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_few_rows_that_do_not_fit_are_flagged(fp8):
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    p = Paged([6, 40], 2, 128, fp8, seed=46)
    q = p.rows(12, 4).cuda()
    for offsets, most, left in (([0, 7, 12], 7, slice(0, 7)), ([0, 6, 12], 5, slice(0, 12)), ([-2, 3, 12], 9, slice(0, 3))):
        out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        cu = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        p.cache.skv_prefill_attn_window(1, q, cu, p.table_dev, p.lens_dev, out, most, 30, 4)
        assert p.cache.skv_get_status() == SKV_ERR_BOUNDS
        assert bool((out[left] == 7.0).all())
        assert left.stop == 12 or bool((out[left.stop:] != 7.0).any())
