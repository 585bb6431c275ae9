"""Attention over a sliding window with sinks, one token per sequence and chunks of tokens, against a 64-bit statement of
it: every kernel variant, lengths around pages and windows, tokens and pages that nobody sees holding garbage."""
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 128), (4, 4, 128), (8, 1, 128), (6, 2, 128), (6, 2, 64), (4, 4, 64), (16, 2, 64)]
LENS = [0, 1, 15, 16, 17, 31, 33, 64, 100, 257, 700, 1500]
WINDOWS = [(1, 0), (1, 1), (16, 0), (17, 5), (100, 4), (333, 70), (5000, 3), (2147483647, 2147483647)]


class Paged:
    """A cache whose sequences hold drawn K, V rows; k[b], v[b]: what the attention is to see of them."""

    def __init__(self, lens, hkv, d, fp8=False, seed=0, spare=3, magnitude=1.0, r=(0, 0)):
        import paper_2604_22782_b200 as skv
        g = torch.Generator().manual_seed(seed)
        self.lens, self.d, self.fp8 = list(lens), d, fp8
        self.table, total = ref.paged(lens, g, spare=spare)
        self.cache = skv.SkvCache(list(r), hkv, d, 16, total, allocate=True, fp8=fp8)
        # pages hold NaN (bf16) / the NaN code with NaN scales (FP8) until something is stored
        if fp8:
            self.cache.pool[256:].fill_(0x7F)
        else:
            self.cache.pool[256:].view(torch.int16).fill_(0x7FC1)
        self.k, self.v, slots = [], [], []
        for b, n in enumerate(self.lens):
            self.k.append((torch.randn(n, hkv, d, generator=g) * magnitude).bfloat16())
            self.v.append((torch.randn(n, hkv, d, generator=g) * magnitude).bfloat16())
            slots.append(ref.slots_of(self.table, b, torch.arange(n)))
        slots = torch.cat(slots).cuda()
        self.cache.skv_append(0, torch.cat(self.k).cuda(), torch.cat(self.v).cuda(), slots)
        if fp8:
            n = slots.numel()
            codes = [torch.empty(n, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
            scales = [torch.empty(n, hkv, dtype=torch.float32, device="cuda") for _ in range(2)]
            self.cache.skv_gather_fp8(0, slots, *codes, *scales)
            back = [(c.view(torch.float8_e4m3fn).double() * s.double()[..., None]).cpu() for c, s in zip(codes, scales)]
            self.k, self.v = (list(torch.split(x, self.lens)) for x in back)
        self.table_dev = self.table.cuda()
        self.lens_dev = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.g = g

    def rows(self, n, hq):
        return torch.randn(n, hq, self.d, generator=self.g).bfloat16()

    def forget(self, first, window, sinks):
        """What the rows from position first[b] on do not see is overwritten with NaN, and pages with nothing else are
        taken out of the table."""
        gone, table = [], self.table.clone()
        for b, n in enumerate(self.lens):
            lo = max(0, first[b] - window + 1)
            t = torch.arange(min(sinks, n), max(min(sinks, n), min(lo, n)))
            gone.append(ref.slots_of(self.table, b, t))
            for p in range(table.shape[1]):
                if all(sinks <= x < lo or x >= n for x in range(16 * p, 16 * p + 16)):
                    table[b, p] = 1 << 30 if p % 2 else -1
        gone = torch.cat(gone)
        if gone.numel() and not self.fp8:
            bad = torch.full((gone.numel(),) + self.k[0].shape[1:], float("nan"), dtype=torch.bfloat16, device="cuda")
            self.cache.skv_append(0, bad, bad, gone.cuda())
        self.table_dev = table.cuda()


def check(got, want, what):
    out, size, reach, n, fp8, v_max = want
    tol = ref.attention_tolerance(out, size, reach, n, fp8, v_max)
    err = (got.double().cpu() - out).abs()
    assert bool((err <= tol).all()), f"{what}: {(err / tol.clamp(min=1e-30)).max().item():.2f} of what rounding allows"


def decode(p, q, window, sinks, layer=1, scale=0.0, **setup):
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(len(p.lens), q.shape[1]), dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_window(layer, q.cuda(), p.table_dev, p.lens_dev, out, ws, window, sinks, scale=scale)
    torch.cuda.synchronize()
    return out


def check_decode(p, q, out, window, sinks, scale=None):
    for b, n in enumerate(p.lens):
        want = ref.attention(q[b:b + 1], p.k[b], p.v[b], torch.tensor([n - 1]), window, sinks, scale)
        v_max = float(p.v[b].double().abs().max()) if n else 0.0
        check(out[b:b + 1], want + (min(n, window + sinks), p.fp8, v_max), f"length {n}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_decode_every_length(hq, hkv, d, window, sinks, fp8):
    p = Paged(LENS, hkv, d, fp8, seed=window % 97 + sinks % 89)
    q = p.rows(len(LENS), hq)
    p.forget([n - 1 for n in LENS], window, sinks)
    out = decode(p, q, window, sinks)
    check_decode(p, q, out, window, sinks)
    assert bool((out[0] == 0).all())                      # no token: a row of zeros
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("worker", [(2, 8, 0, 1), (2, 3, 4, 1), (3, 8, 0, 1), (2, 4, 0, 2)])
@pytest.mark.parametrize("merge", [1, 2])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (4, 4, 64)])
def test_decode_ranges_and_merging(hq, hkv, d, merge, worker):
    """Windows cut into many ranges, with the merge launch and without, and other launch shapes."""
    lens = [4000, 20, 2500, 1, 3999, 0, 1777]
    p = Paged(lens, hkv, d, seed=5)
    p.cache.skv_set_decode_worker(*worker)
    p.cache.skv_set_decode_merge(merge)
    q = p.rows(len(lens), hq)
    for window, sinks in ((1500, 20), (97, 0), (3800, 130)):
        out = decode(p, q, window, sinks)
        check_decode(p, q, out, window, sinks)
    assert p.cache.skv_get_status() == 0


def test_decode_window_longer_than_everything_attends_what_the_plain_call_attends():
    """The same tokens, summed in another order: both within what rounding allows of the same 64-bit result."""
    lens = [300, 1000, 5, 64]
    p = Paged(lens, 2, 128, seed=8)
    q = p.rows(len(lens), 8)
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(4, 8), dtype=torch.uint8, device="cuda")
    plain = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn(1, q.cuda(), p.table_dev, p.lens_dev, plain, ws)
    check_decode(p, q, plain, 1000, 0)
    for window, sinks in ((1000, 0), (1 << 30, 7), (998, 2)):
        check_decode(p, q, decode(p, q, window, sinks), 1000, 0)


def test_decode_infinities_and_lowest_values_outside_the_window():
    lens = [200]
    p = Paged(lens, 2, 128, seed=9)
    window, sinks = 50, 3
    for value in (float("inf"), float("-inf"), torch.finfo(torch.bfloat16).min):
        hidden = ref.slots_of(p.table, 0, torch.arange(sinks, 150)).cuda()
        bad = torch.full((hidden.numel(), 2, 128), value, dtype=torch.bfloat16, device="cuda")
        p.cache.skv_append(0, bad, bad, hidden)
        q = p.rows(1, 8)
        check_decode(p, q, decode(p, q, window, sinks), window, sinks)


def test_decode_scale_and_order_of_sums_repeat():
    lens = [900, 33, 2000]
    p = Paged(lens, 2, 128, seed=10)
    q = p.rows(3, 8)
    first = decode(p, q, 700, 4, scale=0.02)
    check_decode(p, q, first, 700, 4, scale=0.02)
    for _ in range(20):
        assert torch.equal(decode(p, q, 700, 4, scale=0.02), first)


def test_decode_large_batch_in_pieces():
    lens = [(7 * b) % 50 for b in range(5000)]
    p = Paged(lens, 1, 64, seed=11)
    q = p.rows(len(lens), 2)
    out = decode(p, q, 13, 2)
    for b in list(range(0, 30)) + list(range(4080, 4110)) + [4999]:
        want = ref.attention(q[b:b + 1], p.k[b], p.v[b], torch.tensor([lens[b] - 1]), 13, 2)
        check(out[b:b + 1], want + (15, False, 0.0), f"sequence {b}")
    assert p.cache.skv_get_status() == 0


def test_decode_pages_beyond_four_gigabytes():
    import paper_2604_22782_b200 as skv
    pages, hkv, d, n = 70000, 16, 128, 100                # 128 KB a page: 9.2 GB
    cache = skv.SkvCache([0], hkv, d, 16, pages, allocate=True)
    g = torch.Generator().manual_seed(3)
    table = torch.tensor([[69999, 5, 34000, 66000, 17, 69998, 32768]], dtype=torch.int32)
    k, v = torch.randn(n, hkv, d, generator=g).bfloat16(), torch.randn(n, hkv, d, generator=g).bfloat16()
    cache.skv_append(0, k.cuda(), v.cuda(), ref.slots_of(table, 0, torch.arange(n)).cuda())
    q = torch.randn(2, hkv, d, generator=g).bfloat16()
    ws = torch.empty(cache.skv_decode_workspace_bytes(1, hkv), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out = torch.empty(1, hkv, d, dtype=torch.bfloat16, device="cuda")
    cache.skv_decode_attn_window(0, q[1:].cuda(), table.cuda(), lens, out, ws, 60, 20)
    check(out, ref.attention(q[1:], k, v, torch.tensor([n - 1]), 60, 20) + (n, False, 0.0), "decode")
    rows = torch.empty(2, hkv, d, dtype=torch.bfloat16, device="cuda")
    cache.skv_prefill_attn_window(0, q.cuda(), torch.tensor([0, 2], dtype=torch.int32, device="cuda"), table.cuda(), lens, rows, 2, 60, 20)
    check(rows, ref.attention(q, k, v, torch.tensor([n - 2, n - 1]), 60, 20) + (n, False, 0.0), "chunk")
    assert cache.skv_get_status() == 0


def test_decode_captured_and_replayed_with_other_inputs():
    """A captured call reads lengths, tables and queries at replay; two graphs share one workspace in turn."""
    lens = [600, 40, 1300]
    p = Paged(lens, 2, 128, seed=12)
    q, q2 = p.rows(3, 8), p.rows(3, 8)
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(3, 8), dtype=torch.uint8, device="cuda")
    qd, out = q.cuda(), torch.empty(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(s):
        for merge in (1, 2):
            p.cache.skv_set_decode_merge(merge)
            p.cache.skv_decode_attn_window(1, qd, p.table_dev, p.lens_dev, out, ws, 500, 4)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                p.cache.skv_decode_attn_window(1, qd, p.table_dev, p.lens_dev, out, ws, 500, 4)
            graphs.append(g)
    for x in (q, q2, q):
        for g in graphs:
            qd.copy_(x)
            out.fill_(float("nan"))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            check_decode(p, x, out, 500, 4)


def test_decode_two_streams_with_a_workspace_each():
    lens = [3000, 2000, 100, 1500]
    p = Paged(lens, 2, 128, seed=13)
    qs = [p.rows(4, 8) for _ in range(2)]
    streams, outs, works, qd = [torch.cuda.Stream() for _ in range(2)], [], [], [q.cuda() for q in qs]
    for _ in range(2):
        works.append(torch.empty(p.cache.skv_decode_workspace_bytes(4, 8), dtype=torch.uint8, device="cuda"))
        outs.append(torch.empty(4, 8, 128, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            p.cache.skv_decode_attn_window(1, qd[i], p.table_dev, p.lens_dev, outs[i], works[i], 900, 4, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        check_decode(p, qs[i], outs[i], 900, 4)


def chunk(p, q, q_lens, window, sinks, layer=1, scale=0.0, behind=5):
    """The call with rows behind the last sequence's, which have to stay as they were."""
    cu = torch.tensor([0] + torch.tensor(q_lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
    rows = torch.cat((q, torch.zeros(behind, *q.shape[1:], dtype=torch.bfloat16))).cuda()
    out = torch.full(rows.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_window(layer, rows, cu, p.table_dev, p.lens_dev, out, max(1, max(q_lens)), window, sinks, scale=scale)
    torch.cuda.synchronize()
    assert bool((out[len(q):] == 7.0).all())
    return out[:len(q)]


def check_chunk(p, q, q_lens, out, window, sinks, scale=None):
    row = 0
    for b, (n, m) in enumerate(zip(p.lens, q_lens)):
        want = ref.attention(q[row:row + m], p.k[b], p.v[b], torch.arange(n - m, n), window, sinks, scale)
        v_max = float(p.v[b].double().abs().max()) if n else 0.0
        check(out[row:row + m], want + (n, p.fp8, v_max), f"length {n}, {m} rows")
        row += m


CHUNK_LENS = [1, 15, 16, 17, 65, 129, 300, 700, 260, 0]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_chunk_whole_prompts(hq, hkv, d, window, sinks, fp8):
    p = Paged(CHUNK_LENS, hkv, d, fp8, seed=window % 83 + sinks % 79)
    q = p.rows(sum(CHUNK_LENS), hq)
    out = chunk(p, q, CHUNK_LENS, window, sinks)
    check_chunk(p, q, CHUNK_LENS, out, window, sinks)
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 128), (6, 2, 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 0), (64, 3), (300, 17), (129, 200)])
def test_chunk_behind_a_history_that_was_given_back(hq, hkv, d, window, sinks, fp8):
    """The last rows of longer sequences; what none of them sees is NaN or not in the table any more."""
    lens, q_lens = [900, 33, 128, 2049, 5, 300], [100, 33, 0, 513, 1, 17]
    p = Paged(lens, hkv, d, fp8, seed=21)
    q = p.rows(sum(q_lens), hq)
    p.forget([n - m for n, m in zip(lens, q_lens)], window, sinks)
    out = chunk(p, q, q_lens, window, sinks)
    check_chunk(p, q, q_lens, out, window, sinks)
    assert p.cache.skv_get_status() == 0


def test_chunk_of_one_row_is_the_decode_call():
    lens = [900, 33, 128, 2049, 5, 300]
    p = Paged(lens, 2, 128, seed=22)
    q = p.rows(6, 8)
    a, b = chunk(p, q, [1] * 6, 100, 4), decode(p, q, 100, 4)
    check_chunk(p, q, [1] * 6, a, 100, 4)
    check_decode(p, q, b, 100, 4)


def test_chunk_many_short_sequences_beside_a_long_one():
    lens = [1 + b % 3 for b in range(300)] + [1000] + [2] * 40
    q_lens = [1] * 300 + [900] + [2] * 40
    p = Paged(lens, 1, 128, seed=23)
    q = p.rows(sum(q_lens), 4)
    check_chunk(p, q, q_lens, chunk(p, q, q_lens, 200, 4), 200, 4)
    assert p.cache.skv_get_status() == 0


def test_chunk_repeats_bit_for_bit():
    p = Paged(CHUNK_LENS, 2, 128, seed=24)
    q = p.rows(sum(CHUNK_LENS), 8)
    first = chunk(p, q, CHUNK_LENS, 100, 4, scale=0.3)
    check_chunk(p, q, CHUNK_LENS, first, 100, 4, scale=0.3)
    for _ in range(40):
        assert torch.equal(chunk(p, q, CHUNK_LENS, 100, 4, scale=0.3), first)


@pytest.mark.parametrize("fp8", [False, True])
def test_lengths_that_do_not_fit_are_flagged(fp8):
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    p = Paged([70, 40], 2, 128, fp8, seed=25)
    q = p.rows(110, 4).cuda()
    cu = torch.tensor([0, 71, 110], dtype=torch.int32, device="cuda")          # more rows than tokens
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_window(1, q, cu, p.table_dev, p.lens_dev, out, 71, 30, 4)
    assert p.cache.skv_get_status() == SKV_ERR_BOUNDS
    assert bool((out[:71] == 7.0).all()) and bool((out[71:] != 7.0).any())
    table = p.table_dev.clone()
    table[1, 2] = 1 << 20                                                       # a page id beyond the pool, inside the window
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(2, 4), dtype=torch.uint8, device="cuda")
    o = torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_window(1, q[:2], table, p.lens_dev, o, ws, 8, 0)
    assert p.cache.skv_get_status() == SKV_ERR_BOUNDS
    p.cache.skv_decode_attn_window(1, q[:2], p.table_dev[:, :2].contiguous(), p.lens_dev, o, ws, 8, 0)   # longer than the row
    assert p.cache.skv_get_status() == SKV_ERR_BOUNDS


def test_refusals():
    from paper_2604_22782_b200.binding import SKV_ERR_ARG, SKV_ERR_LAYER, SKV_ERR_NOMEM, SKV_ERR_UNSUPPORTED, SkvError
    p = Paged([70, 40], 2, 128, seed=26)
    q, out = p.rows(2, 4).cuda(), torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(p.cache.skv_decode_workspace_bytes(2, 4), dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    before = p.cache.skv_launch_count()

    def refused(status, layer=1, q=q, out=out, ws=ws, window=8, sinks=0):
        with pytest.raises(SkvError) as e:
            p.cache.skv_decode_attn_window(layer, q, p.table_dev, p.lens_dev, out, ws, window, sinks)
        assert e.value.status == status
        if status != SKV_ERR_NOMEM:
            with pytest.raises(SkvError) as e:
                p.cache.skv_prefill_attn_window(layer, q, cu, p.table_dev, p.lens_dev, out, 1, window, sinks)
            assert e.value.status == status

    refused(SKV_ERR_ARG, window=0)
    refused(SKV_ERR_ARG, window=-5)
    refused(SKV_ERR_ARG, sinks=-1)
    refused(SKV_ERR_LAYER, layer=2)
    refused(SKV_ERR_NOMEM, ws=ws[:-256])
    odd = torch.empty(2, 3, 128, dtype=torch.bfloat16, device="cuda")
    refused(SKV_ERR_UNSUPPORTED, q=odd, out=torch.empty_like(odd))
    with pytest.raises(ValueError):
        p.cache.skv_decode_attn_window(1, q, p.table_dev, p.lens_dev, out, ws, 1 << 32, 0)
    with pytest.raises(ValueError):
        p.cache.skv_decode_attn_window(1, q.transpose(0, 1), p.table_dev, p.lens_dev, out, ws, 8, 0)
    assert p.cache.skv_launch_count() == before and p.cache.skv_get_status() == 0
