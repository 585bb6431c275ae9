"""The page index, the selection of pages and attention over listed pages, each against a plain statement of it, and the
four calls of a layer together."""
import math
import random

import pytest
import torch

import pages_reference as pages
import serving_reference as ref
from test_gpu_window import Paged

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 128), (4, 4, 128), (8, 1, 128), (6, 2, 128), (6, 2, 64), (4, 4, 64), (16, 2, 64)]
LENS = [0, 1, 15, 16, 17, 31, 33, 64, 100, 257, 700, 1500]


def index_of(cache, layers=1):
    """Memory for the cache's index, and per owner layer its codes [page][head][2][D] and scales [page][head]."""
    memory = torch.empty(cache.skv_page_index_bytes(), dtype=torch.uint8, device="cuda")
    cache.skv_set_page_index(memory)
    n, h, d = cache.max_pages, cache.kv_heads, cache.head_dim
    codes = -(-n * h * 2 * d // 256) * 256
    layer = codes + -(-n * h * 4 // 256) * 256
    assert memory.numel() == layers * layer
    return memory, [(memory[i * layer:][:n * h * 2 * d].view(torch.int8).view(n, h, 2, d),
                     memory[i * layer + codes:][:n * h * 4].view(torch.float32).view(n, h)) for i in range(layers)]


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(got, want, what):
    """serving_reference's bounds.  A tile at a time on FP8 pages: queries are two E4M3 terms times a power of two (exact, but for elements
    below 2^-9 of the row's largest: 2^-17 of that at most), probabilities times V scale over c are f16, as they are where a row is taken at
    a time."""
    out, size, reach, n, fp8, v_max = want
    tol = ref.attention_tolerance(out, size, reach, n, fp8, v_max)
    err = (got.double().cpu() - out).abs()
    assert bool((err <= tol).all()), f"{what}: {(err / tol.clamp(min=1e-30)).max().item():.2f} of what rounding allows"


# ---- the index -----------------------------------------------------------------------------------------------------
def check_index(p, codes, scales, full_from, full_to):
    """Entries of pages [full_from[b], full_to[b]) are as stated; everything else is as it was (zero)."""
    want_codes, want_scales = torch.zeros(codes.shape, dtype=torch.int8), torch.zeros(scales.shape)
    for b in range(len(p.lens)):
        for j in range(full_from[b], full_to[b]):
            for h in range(codes.shape[1]):
                rows = p.k[b][16 * j:16 * j + 16, h]
                want_codes[p.table[b, j], h], want_scales[p.table[b, j], h] = pages.index_entry(rows)
    assert torch.equal(codes.cpu(), want_codes)
    assert torch.equal(scales.cpu(), want_scales)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hkv,d", [(2, 128), (1, 64), (3, 128), (8, 64)])
@pytest.mark.parametrize("share", [0.0, 0.4, 1.0])
def test_index_of_new_tokens(hkv, d, fp8, share):
    p = Paged(LENS, hkv, d, fp8, seed=hkv + d, r=(0, 0))
    if fp8:                                                # (what was stored, in fp32: code value x scale, one rounding)
        p.k = [k.float() for k in p.k]
    _, [(codes, scales)] = index_of(p.cache)
    new = [int(n * share) for n in LENS]
    cu = [sum(new[:b]) for b in range(len(new) + 1)]
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu_q_lens=i32(cu), max_q_len=max(max(new), 1))
    check_index(p, codes, scales, [(n - a) // 16 for n, a in zip(LENS, new)], [n // 16 for n in LENS])
    launches = p.cache.skv_launch_count()
    p.cache.skv_index_pages(1, p.table_dev, p.lens_dev)   # a layer that keeps nothing
    assert p.cache.skv_launch_count() == launches and p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_index_of_one_token_each(fp8):
    lens = [0, 1, 16, 32, 33, 48, 15, 160]
    p = Paged(lens, 2, 128, fp8, seed=3)
    p.k = [k.float() for k in p.k]
    _, [(codes, scales)] = index_of(p.cache)
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev)
    check_index(p, codes, scales, [max(n - 1, 0) // 16 for n in lens], [n // 16 for n in lens])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_index_with_room_for_many_more_tokens(fp8):
    """A bound on the new tokens far above what there are, so that a CTA goes through its items in several rounds."""
    lens = [700, 0, 33, 1000, 64]
    p = Paged(lens, 3, 64, fp8, seed=7)
    p.k = [k.float() for k in p.k]
    _, [(codes, scales)] = index_of(p.cache)
    table = torch.full((5, 9000), -1, dtype=torch.int32)
    table[:, :p.table.shape[1]] = p.table
    cu = [sum(lens[:b]) for b in range(6)]
    p.cache.skv_index_pages(0, table.cuda(), p.lens_dev, cu_q_lens=i32(cu), max_q_len=144000)
    check_index(p, codes, scales, [0] * 5, [n // 16 for n in lens])
    assert p.cache.skv_get_status() == 0


def test_index_of_unusual_keys():
    """Zeros, next to nothing, one large value, the largest finite ones, infinities, NaN: head by head."""
    import paper_2604_22782_b200 as skv
    p = Paged([160], 1, 128, seed=4)
    _, [(codes, scales)] = index_of(p.cache)
    k = torch.randn(160, 1, 128, generator=p.g).bfloat16()
    k[0:16] = 0
    k[16:32] = 1e-35
    k[32:48] *= 2.0 ** -80
    k[48:64, 0, 5] = 3.0e38
    k[64:80] = torch.finfo(torch.bfloat16).min
    k[80, 0, 127] = math.inf
    k[100, 0, 0] = -math.inf
    k[119, 0, 64] = math.nan
    k[128:144] = -k[128:144].abs()
    p.cache.skv_append(0, k.cuda(), k.cuda(), ref.slots_of(p.table, 0, torch.arange(160)).cuda())
    p.k = [k]
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu_q_lens=i32([0, 160]), max_q_len=160)
    check_index(p, codes, scales, [0], [10])
    assert isinstance(p.cache, skv.SkvCache) and p.cache.skv_get_status() == 0


def test_index_refuses_on_the_device():
    from paper_2604_22782_b200 import binding as B
    p = Paged([64, 64, 64, 64], 2, 64, seed=5)
    _, [(codes, scales)] = index_of(p.cache)
    p.k = [k.float() for k in p.k]
    cu = i32([0, 64, 128, 192, 256])
    p.cache.skv_index_pages(0, p.table_dev, i32([64, 63, 64, 65 * 16]), cu_q_lens=cu, max_q_len=64)      # fewer tokens than rows; too long
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    check_index(p, codes, scales, [0] * 4, [4, 0, 4, 0])
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu_q_lens=cu, max_q_len=63)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    p.table[1, 2], p.table[2, 0] = -1, 1 << 20
    p.cache.skv_index_pages(0, p.table.cuda(), p.lens_dev, cu_q_lens=cu, max_q_len=64)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS


# ---- the selection -------------------------------------------------------------------------------------------------
class Indexed:
    """A cache of sequences whose index holds drawn codes."""

    def __init__(self, lens, hkv, d, seed=0, kind="drawn"):
        import paper_2604_22782_b200 as skv
        g = self.g = torch.Generator().manual_seed(seed)
        self.lens = list(lens)
        self.table, total = ref.paged(lens, g, spare=2)
        self.cache = skv.SkvCache([0, 0], hkv, d, 16, total, allocate=True)
        self.memory, [(codes, scales)] = index_of(self.cache)
        c = torch.randint(-127, 128, codes.shape, generator=g, dtype=torch.int32)
        s = torch.rand(scales.shape, generator=g) + 0.1
        if kind == "ties":                                 # few different scores
            c, s = (c > 120).int() * 3, torch.full(scales.shape, 0.5)
        if kind == "equal":
            s = torch.zeros(scales.shape)
        if kind == "wild":
            s[torch.rand(scales.shape, generator=g) < 0.2] = math.inf
        self.codes, self.scales = c.to(torch.int8), s
        codes.copy_(self.codes)
        scales.copy_(self.scales)
        self.table_dev, self.lens_dev = self.table.cuda(), i32(self.lens)

    def select(self, q, top, first, last, new=None, most=1, run=1, width=None, layer=1):
        import paper_2604_22782_b200 as skv
        per = -(-most // run)
        width = width or skv.skv_page_list_width(top, first, last, run)
        lists = torch.full((len(self.lens) * per, self.cache.kv_heads, width), 77, dtype=torch.int32, device="cuda")
        counts = torch.full((len(self.lens) * per, self.cache.kv_heads), 77, dtype=torch.int32, device="cuda")
        cu = None if new is None else i32([sum(new[:b]) for b in range(len(new) + 1)])
        self.cache.skv_select_pages(layer, q.cuda(), self.table_dev, self.lens_dev, lists, counts, top, first, last, cu_q_lens=cu, max_q_len=most, run=run)
        return lists.cpu(), counts.cpu()

    def check(self, q, lists, counts, top, first, last, new=None, most=1, run=1):
        per, hkv = -(-most // run), self.cache.kv_heads
        for b, n in enumerate(self.lens):
            rows = [1 if n else 0] * len(self.lens) if new is None else new
            start = b if new is None else sum(new[:b])
            for r in range(per):
                a = min(rows[b], (r + 1) * run) - r * run
                for h in range(hkv):
                    want = []
                    if a > 0:
                        p0 = n - rows[b] + r * run
                        ids = self.table[b].clamp(min=0).long()
                        group = q.shape[1] // hkv
                        mine = q[start + r * run:start + r * run + a, h * group:(h + 1) * group]
                        want = pages.page_list(pages.scores(mine, self.codes[ids, h], self.scales[ids, h]), p0, p0 + a - 1, top, first, last)
                    got = lists[b * per + r, h].tolist()
                    assert counts[b * per + r, h] == len(want), (n, r, h)
                    assert got == want + [-1] * (len(got) - len(want)), (n, r, h)
        assert self.cache.skv_get_status() == 0


@pytest.mark.parametrize("kind", ["drawn", "ties", "equal", "wild"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("top,first,last", [(0, 0, 1), (0, 2, 3), (1, 0, 1), (5, 1, 2), (31, 3, 1), (64, 1, 20), (500, 1, 1)])
def test_selection_for_one_row_each(hq, hkv, d, top, first, last, kind):
    p = Indexed(LENS, hkv, d, seed=top + first, kind=kind)
    q = torch.randn(len(LENS), hq, d, generator=p.g).bfloat16()
    lists, counts = p.select(q, top, first, last)
    p.check(q, lists, counts, top, first, last)


@pytest.mark.parametrize("hq,hkv,d,run", [(8, 2, 128, 32), (8, 2, 128, 5), (8, 2, 128, 4), (6, 2, 128, 2), (4, 4, 128, 128), (4, 4, 128, 7), (8, 1, 128, 16), (6, 2, 64, 42), (6, 2, 64, 1),
                                          (6, 2, 64, 4), (4, 4, 64, 33), (16, 2, 64, 2)])
@pytest.mark.parametrize("kind", ["drawn", "ties", "wild"])
def test_selection_for_runs(hq, hkv, d, run, kind):
    lens, new = [0, 1, 40, 300, 1201, 2000], [0, 1, 40, 77, 150, 1]
    p = Indexed(lens, hkv, d, seed=run, kind=kind)
    q = torch.randn(sum(new), hq, d, generator=p.g).bfloat16()
    for top, first, last in ((9, 1, 2), (40, 0, 1), (0, 1, 4)):
        lists, counts = p.select(q, top, first, last, new, 150, run)
        p.check(q, lists, counts, top, first, last, new, 150, run)


@pytest.mark.parametrize("batch", [75, 250, 260])
def test_selection_of_many_sequences(batch):
    """More segments than SMs, with lengths all over, equal ones among them: longest first, and beyond 256 as they come."""
    lens = [(37 * b * b + 11 * b) % 900 for b in range(batch)]
    lens[3], lens[batch // 2], lens[batch - 1] = 0, lens[1], 900
    p = Indexed(lens, 2, 64, seed=batch)
    q = torch.randn(batch, 4, 64, generator=p.g).bfloat16()
    lists, counts = p.select(q, 9, 1, 2)
    p.check(q, lists, counts, 9, 1, 2)


@pytest.mark.parametrize("batch", [1, 3, 40])
def test_selection_in_long_caches(batch):
    """Thousands of pages: a cluster of CTAs for a segment, and one alone."""
    lens = [40000 - 611 * b for b in range(batch)]
    p = Indexed(lens, 2, 64, seed=batch)
    q = torch.randn(batch, 4, 64, generator=p.g).bfloat16()
    for top in (100, 1999):
        lists, counts = p.select(q, top, 1, 8)
        p.check(q, lists, counts, top, 1, 8)
    if batch == 3:                                            # many columns
        new = [20, 9, 31]
        q = torch.randn(sum(new), 4, 64, generator=p.g).bfloat16()
        for run in (9, 31):
            lists, counts = p.select(q, 300, 2, 3, new, 31, run)
            p.check(q, lists, counts, 300, 2, 3, new, 31, run)


def test_selection_with_unusual_queries():
    p = Indexed([700] * 6, 2, 128, seed=8)
    q = torch.randn(6, 8, 128, generator=p.g).bfloat16()
    q[0] = 0
    q[1] *= 2.0 ** -110
    q[2, 3, 7], q[2, 4, 9] = math.nan, math.inf
    q[3] = math.nan
    q[4, 0, 0] = torch.finfo(torch.bfloat16).max
    lists, counts = p.select(q, 9, 1, 2)
    p.check(q, lists, counts, 9, 1, 2)


def test_selection_refuses_on_the_device():
    from paper_2604_22782_b200 import binding as B
    p = Indexed([400, 400, 400], 2, 64, seed=9)
    q = torch.randn(30, 4, 64, generator=p.g).bfloat16()
    before = p.lens
    p.lens_dev = i32([400, 400, 401 * 16])
    lists, counts = p.select(q, 4, 1, 1, [10, 10, 10], 10, 10)
    assert counts[2].tolist() == [0, 0] and bool((lists[2] == -1).all()) and p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    p.lens, p.lens_dev = before, i32(before)
    lists, counts = p.select(q, 4, 1, 1, [10, 10, 10], 9, 9)                       # more rows than the bound
    assert bool((counts == 0).all()) and p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    lists, counts = p.select(q[:3], 4, 1, 1)
    p.check(q[:3], lists, counts, 4, 1, 1)
    p.table_dev[1, 3] = -5                                                          # scored as page 0
    p.select(q[:3], 4, 1, 1)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    p.table_dev = p.table.cuda()
    p.lens_dev = i32([400, 16 * p.table.shape[1] + 5, 400])                          # cut to the row
    lists, counts = p.select(q[:3], 4, 1, 1)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    p.lens[1] = 400
    p.check(q[:3], lists, counts, 4, 1, 1)


# ---- attention -----------------------------------------------------------------------------------------------------
def some_lists(rng, page_counts, hkv, width, keep_last=True):
    """Per sequence (or run) and head a random choice of its pages in a random order; -7 behind the last."""
    lists = torch.full((len(page_counts), hkv, width), -7, dtype=torch.int32)
    counts = torch.zeros((len(page_counts), hkv), dtype=torch.int32)
    for i, m in enumerate(page_counts):
        for h in range(hkv):
            mine = rng.sample(range(m), min(m, rng.randint(0, width)))
            if keep_last and m and width and m - 1 not in mine:
                mine = mine[:width - 1] + [m - 1]
            rng.shuffle(mine)
            lists[i, h, :len(mine)], counts[i, h] = torch.tensor(mine, dtype=torch.int32), len(mine)
    return lists, counts


def check_rows(p, q, out, lists, counts, rows_of, scale=None):
    """rows_of[i] = (sequence, first row of q, positions) of list i."""
    hkv = lists.shape[1]
    group = q.shape[1] // hkv
    for i, (b, row, pos) in enumerate(rows_of):
        for h in range(hkv):
            mine = slice(row, row + len(pos)), slice(h * group, (h + 1) * group)
            want = pages.attention(q[mine], p.k[b][:, h], p.v[b][:, h], torch.tensor(pos), lists[i, h, :counts[i, h]].tolist(), scale)
            v_max = float(p.v[b].double().abs().max()) if p.lens[b] else 0.0
            check(out[mine], want + (16 * int(counts[i, h]), p.fp8, v_max), f"list {i} head {h}")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("width", [1, 7, 100])
def test_decode_over_listed_pages(hq, hkv, d, width, fp8):
    p = Paged(LENS, hkv, d, fp8, seed=width)
    q = p.rows(len(LENS), hq)
    lists, counts = some_lists(random.Random(width), [-(-n // 16) for n in LENS], hkv, width)
    counts[5, 0] = 0
    counts[6, hkv - 1] = -3
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(1, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    counts = counts.clamp(min=0)
    check_rows(p, q, out, lists, counts, [(b, b, [n - 1]) for b, n in enumerate(LENS)])
    assert bool((out[0] == 0).all()) and bool((out[5, :hq // hkv] == 0).all()) and p.cache.skv_get_status() == 0


@pytest.mark.parametrize("variant", [1, 2])
def test_decode_variants_and_scale(variant):
    p = Paged([900, 40], 4, 128, seed=variant)
    p.cache.skv_set_decode_variant(variant)
    q = p.rows(2, 4)
    lists, counts = some_lists(random.Random(variant), [57, 3], 4, 40)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, scale=0.3)
    check_rows(p, q, out, lists, counts, [(0, 0, [899]), (1, 1, [39])], scale=0.3)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("batch", [1, 2, 5, 10, 30, 60, 150])
def test_decode_launch_shapes(batch, fp8):
    """One segment to many: clusters of every size, long lists, warps without pages."""
    lens = [6000 if b == 0 else 200 + 37 * b % 1000 for b in range(batch)]
    p = Paged(lens, 2, 128, fp8, seed=batch)
    q = p.rows(batch, 8)
    lists, counts = some_lists(random.Random(batch), [-(-n // 16) for n in lens], 2, 300)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(b, b, [n - 1]) for b, n in enumerate(lens)])
    again = torch.empty_like(out)
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("batch,fp8", [(60, False), (112, False), (240, False), (112, True), (240, True)])
def test_decode_of_more_segments_than_sms(batch, fp8):
    """A segment to a CTA of four warps, or to two, and three or four of these to an SM; lists of a few pages to many."""
    lens = [1300 if b % 7 == 0 else 5 + 61 * b % 900 for b in range(batch)]
    p = Paged(lens, 2, 128, fp8, seed=batch)
    q = p.rows(batch, 8)
    lists, counts = some_lists(random.Random(batch), [-(-n // 16) for n in lens], 2, 80)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(b, b, [n - 1]) for b, n in enumerate(lens)])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_a_page_listed_twice_counts_twice(fp8):
    p = Paged([100, 333], 2, 128, fp8, seed=4)
    lists = torch.tensor([[[2, 2, 6], [6, 0, 6]], [[20, 3, 20], [7, 7, 7]]], dtype=torch.int32)
    counts = torch.full((2, 2), 3, dtype=torch.int32)
    q = p.rows(2, 8)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(0, 0, [99]), (1, 1, [332])])
    rows = p.rows(2 * 32, 8)
    runs = [(b, 32 * b, list(range(n - 32, n))) for b, n in enumerate(p.lens)]
    for variant in (1, 2):
        p.cache.skv_set_prefill_variant(variant)
        out = torch.empty(rows.shape, dtype=torch.bfloat16, device="cuda")
        p.cache.skv_prefill_attn_pages(0, rows.cuda(), i32([0, 32, 64]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, 32, run=32)
        check_rows(p, rows, out, lists, counts, runs)


CHUNKS = [(8, 2, 128, 32), (8, 2, 128, 3), (4, 4, 128, 128), (8, 1, 128, 16), (6, 2, 64, 42), (6, 2, 128, 1), (4, 4, 64, 33), (16, 2, 64, 7), (8, 2, 64, 32)]


def chunk_runs(lens, new, most, run):
    """(sequence, first row of q, positions) of every list."""
    got = []
    for b, (n, a) in enumerate(zip(lens, new)):
        for r in range(-(-most // run)):
            at, end = r * run, min(a, (r + 1) * run)
            got.append((b, sum(new[:b]) + at, list(range(n - a + at, n - a + end))) if at < end else (b, 0, []))
    return got


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("hq,hkv,d,run", CHUNKS)
def test_chunks_over_listed_pages(hq, hkv, d, run, fp8, variant):
    """A row at a time and a tile at a time."""
    lens, new = [0, 1, 40, 300, 1201, 2000, 129], [0, 1, 40, 77, 150, 1, 0]
    p = Paged(lens, hkv, d, fp8, seed=run)
    p.cache.skv_set_prefill_variant(variant)
    q = p.rows(sum(new), hq)
    runs = chunk_runs(lens, new, 150, run)
    lists, counts = some_lists(random.Random(run), [(r[2][-1] // 16 + 1 if r[2] else 0) for r in runs], hkv, 30, keep_last=False)
    held = torch.full((len(q) + run, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")          # rows behind the last stay as they are
    out = held[:len(q)]
    cu = i32([sum(new[:b]) for b in range(len(new) + 1)])
    p.cache.skv_prefill_attn_pages(1, q.cuda(), cu, p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, 150, run=run)
    check_rows(p, q, out, lists, counts, runs)
    assert p.cache.skv_get_status() == 0 and bool((held[len(q):] == 7.0).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
@pytest.mark.parametrize("width,batch", [(7, 1), (20, 1), (60, 9), (200, 1), (200, 9), (200, 30)])
def test_few_lists_in_parts(hq, hkv, d, width, batch, fp8):
    """Two, four or eight CTAs to a list, of which some have no block of it, or none that a row sees a token of."""
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    lens = [3600 - 31 * b for b in range(batch)]
    p = Paged(lens, hkv, d, fp8, seed=width)
    p.cache.skv_set_prefill_variant(2)
    q = p.rows(30 * batch, hq)
    q[7, 1, 3] = math.nan
    runs = chunk_runs(lens, [30] * batch, 30, 30)
    lists, counts = some_lists(random.Random(width), [-(-n // 16) for n in lens], hkv, width)
    counts[0, 1] = 1
    lists[batch - 1, 0, :5], counts[batch - 1, 0] = lens[-1] // 16 - 1 + torch.tensor([0, 1, 1, 1, 1], dtype=torch.int32), 5      # first rows see only the first of them
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    args = 0, q.cuda(), i32(range(0, 30 * batch + 1, 30)), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda()
    p.cache.skv_prefill_attn_pages(*args, out, 30, 30)
    again = torch.empty_like(out)
    p.cache.skv_prefill_attn_pages(*args, again, 30, 30)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    # (where the last page is full the one behind it, listed here, is none of the sequence's: left out, and reported)
    assert p.cache.skv_get_status() == (SKV_ERR_BOUNDS if lens[-1] % 16 == 0 else 0)
    want = torch.zeros(q.shape[:2], dtype=torch.bool)
    want[7, 1] = any(16 * page <= runs[0][2][7] for page in lists[0, 0, :counts[0, 0]].tolist())      # (one that sees nothing gives zeros)
    out = out.cpu()
    assert torch.equal(torch.isnan(out).all(-1), want) and torch.equal(torch.isnan(out).any(-1), want)
    q[7, 1] = 0.0
    p.cache.skv_prefill_attn_pages(0, q.cuda(), *args[2:], again, 30, 30)
    out[7, 1] = again[7, 1].cpu()                             # (that row from a call without the NaN)
    check_rows(p, q, out, lists, counts, runs)


@pytest.mark.parametrize("variant", [1, 2])
def test_hidden_tokens_and_unlisted_pages_may_hold_anything(variant):
    """NaN behind a row's position and in pages that are not listed; page-table entries that are not listed are not read."""
    lens, new = [1000, 333], [20, 7]
    for d, hkv, hq in ((128, 2, 8), (64, 2, 6), (128, 4, 4)):
        p = Paged(lens, hkv, d, seed=d)
        p.cache.skv_set_prefill_variant(variant)
        q = p.rows(27, hq)
        runs = chunk_runs(lens, new, 20, 4)
        rng = random.Random(d)
        some = [sorted(rng.sample(range(n // 16 - 2), 9)) for n in lens]                     # the same for a sequence's runs and heads
        lists = torch.full((len(runs), hkv, 12), -1, dtype=torch.int32)
        counts = torch.zeros((len(runs), hkv), dtype=torch.int32)
        for i, (b, _, pos) in enumerate(runs):
            if pos:
                mine = some[b] + list(range(pos[0] // 16, pos[-1] // 16 + 1))
                lists[i, :, :len(mine)], counts[i] = torch.tensor(mine, dtype=torch.int32), len(mine)
        table = p.table.clone()
        for b, n in enumerate(lens):
            held = set(some[b]) | set(range((n - new[b]) // 16, -(-n // 16)))
            gone = [t for t in range(n) if t // 16 not in held]
            bad = torch.full((len(gone), hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            p.cache.skv_append(0, bad, bad, ref.slots_of(p.table, b, torch.tensor(gone)).cuda())
            for j in range(-(-n // 16)):
                if j not in held:
                    table[b, j] = -1 if j % 2 else 1 << 30
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, 20, 27]), table.cuda(), p.lens_dev, lists.cuda(), counts.cuda(), out, 20, run=4)
        check_rows(p, q, out, lists, counts, runs)
        last = [len(r) for r in (range(20), range(7))]
        ends = [19, 26]
        one = torch.empty(2, hq, d, dtype=torch.bfloat16, device="cuda")
        own = [(max(i for i, r in enumerate(runs) if r[0] == b and r[2])) for b in range(2)]
        p.cache.skv_decode_attn_pages(0, q[ends].cuda(), table.cuda(), p.lens_dev, lists[own].contiguous().cuda(), counts[own].contiguous().cuda(), one)
        check_rows(p, q[ends], one, lists[own], counts[own], [(b, b, [lens[b] - 1]) for b in range(2)])
        assert last == new and p.cache.skv_get_status() == 0


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("hq,hkv,d,run", [(8, 2, 128, 16), (6, 2, 64, 5)])
def test_fp8_codes_of_every_value(hq, hkv, d, run, variant):
    """All 254 finite codes, subnormal ones among them, at scales far apart; a NaN key and a NaN value reach the rows that see them."""
    n, a = 512, 2 * run
    p = Paged([n], hkv, d, True, seed=run)
    p.cache.skv_set_prefill_variant(variant)
    codes = torch.tensor([c for c in range(256) if c & 0x7F != 0x7F], dtype=torch.uint8).view(torch.float8_e4m3fn).float()
    at = torch.randint(0, 254, (n, hkv, d), generator=p.g)
    at[..., 0] = 126                                          # 448: it is the row's largest, so that codes come back as they went in
    size = torch.exp2(torch.randint(-3, 4, (n, hkv, 1), generator=p.g).float())
    v = (codes[at] * size / 64).bfloat16()
    k = (codes[at.flip(0)] * size / 1024).bfloat16()
    slots = ref.slots_of(p.table, 0, torch.arange(n)).cuda()
    p.cache.skv_append(0, k.cuda(), v.cuda(), slots)
    p.k, p.v = [k.double()], [v.double()]                     # (a power of two times a code: exact)
    back = [torch.empty(n, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2)], [torch.empty(n, hkv, device="cuda") for _ in range(2)]
    p.cache.skv_gather_fp8(0, slots, *back[0], *back[1])
    assert torch.equal(back[0][1].cpu().view(torch.float8_e4m3fn).double() * back[1][1].cpu().double()[..., None], v.double())
    q = p.rows(a, hq)
    runs = chunk_runs([n], [a], a, run)
    lists, counts = some_lists(random.Random(run), [n // 16] * 2, hkv, 20)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")

    def attend():
        p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, a, run=run)
        assert p.cache.skv_get_status() == 0
    attend()
    check_rows(p, q, out, lists, counts, runs)
    k[n - 3, 0, 5] = v[n - 2, 1, 7] = math.nan
    p.cache.skv_append(0, k[n - 3:].cuda(), v[n - 3:].cuda(), slots[n - 3:])
    attend()
    nan = torch.isnan(out.cpu())
    group = hq // hkv
    assert bool(nan[a - 3:, :group].all()) and not bool(nan[:a - 3, :group].any())
    assert bool(nan[a - 2:, group:2 * group, 7].all()) and not bool(nan[:a - 16, group:].any())


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("hq,hkv,d,run", [(8, 2, 128, 16), (6, 2, 64, 5)])
def test_fp8_queries_of_every_size(hq, hkv, d, run, variant):
    """Rows of zeros, rows far apart in size and elements far apart within a row.  A query element may be off by 2^-17 of the row's largest at most
    (serving_reference counts 2^-11 of every product): 2^-17 max|q| sum|k| on a score, twice that on what it weighs."""
    n, a = 400, 2 * run
    p = Paged([n], hkv, d, True, seed=d)
    p.cache.skv_set_prefill_variant(variant)
    q = p.rows(a, hq).float()
    q *= torch.exp2(torch.randint(-14, 1, q.shape, generator=p.g).float())
    q *= torch.exp2(torch.tensor([-110.0, -40.0, -3.0, 0.0, 2.0])[torch.randint(0, 5, (a, hq, 1), generator=p.g)])
    q[3] = 0.0
    q = q.bfloat16()
    runs = chunk_runs([n], [a], a, run)
    lists, counts = some_lists(random.Random(run), [n // 16] * 2, hkv, 20)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, a, run=run)
    group = hq // hkv
    for i, (b, row, pos) in enumerate(runs):
        for h in range(hkv):
            mine = slice(row, row + len(pos)), slice(h * group, (h + 1) * group)
            want = pages.attention(q[mine], p.k[0][:, h], p.v[0][:, h], torch.tensor(pos), lists[i, h, :counts[i, h]].tolist())
            tol = ref.attention_tolerance(*want, 16 * int(counts[i, h]), True, float(p.v[0].double().abs().max()))
            far = q[mine].double().abs().amax(2, keepdim=True) * p.k[0][:, h].double().abs().sum(1).max() / math.sqrt(d)
            err = (out[mine].double().cpu() - want[0]).abs()
            assert bool((err <= tol + 2 * 2 ** -17 * far * want[1]).all())
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("d,hkv,hq", [(128, 2, 8), (64, 2, 6)])
def test_fp8_value_scales_far_apart(d, hkv, hq, variant):
    """V rows of zeros, V growing by 2^12 from page to page of a list and falling again, and a huge one that earlier rows must not see."""
    n, a, run = 288, 8, 8
    p = Paged([n], hkv, d, True, seed=d)
    p.cache.skv_set_prefill_variant(variant)
    v = torch.randn(n, hkv, d, generator=p.g)
    for j, e in enumerate([None, -60, -48, -36, -24, -12, 0, 12, 24, 30, 12, 0, -12, -36, None, 0, 0, 0]):
        v[16 * j:16 * j + 16] *= 0.0 if e is None else 2.0 ** e
    v[n - 1] *= 2.0 ** 60
    v = v.bfloat16()
    slots = ref.slots_of(p.table, 0, torch.arange(n)).cuda()
    k = p.k[0].bfloat16()
    p.cache.skv_append(0, k.cuda(), v.cuda(), slots)
    codes, scales = [torch.empty(n, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2)], [torch.empty(n, hkv, device="cuda") for _ in range(2)]
    p.cache.skv_gather_fp8(0, slots, *codes, *scales)
    p.k, p.v = ([(c.view(torch.float8_e4m3fn).double() * x.double()[..., None]).cpu()] for c, x in zip(codes, scales))
    q = p.rows(a, hq)
    runs = chunk_runs([n], [a], a, run)
    for pages_listed in ([0, 14], list(range(9)), [8, 7, 1, 0], list(range(18)), [0, 14, 17], [13, 1, 2, 17]):
        lists = torch.tensor(pages_listed, dtype=torch.int32).expand(1, hkv, -1).contiguous()
        counts = torch.full((1, hkv), len(pages_listed), dtype=torch.int32)
        out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, a, run=run)
        for i in range(a):                                    # row by row: what a row does not see has no part in its bound
            there = [t for j in pages_listed for t in range(16 * j, 16 * j + 16) if t <= n - a + i]
            v_max = float(p.v[0][there].abs().max())
            for h in range(hkv):
                mine = slice(i, i + 1), slice(h * hq // hkv, (h + 1) * hq // hkv)
                want = pages.attention(q[mine], p.k[0][:, h], p.v[0][:, h], torch.tensor([n - a + i]), pages_listed)
                check(out[mine], want + (len(there), True, v_max), f"pages {pages_listed} row {i} head {h}")
    assert p.cache.skv_get_status() == 0 and len(runs) == 1


@pytest.mark.parametrize("fp8", [False, True])
def test_lists_that_do_not_fit_are_reported(fp8):
    from paper_2604_22782_b200 import binding as B
    p = Paged([100, 100], 2, 128, fp8, seed=2)
    q = p.rows(2, 8)
    lists = i32([[[3, 7, 0, -1], [0, 1, 2, 3]], [[6, 1, 1 << 30, 2], [5, 4, 3, 2]]])
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists, i32([[4, 4], [4, 9]]), out)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    left = torch.tensor([[[3, 0, 0, 0], [0, 1, 2, 3]], [[6, 1, 2, 0], [5, 4, 3, 2]]])
    check_rows(p, q, out, left, torch.tensor([[2, 4], [3, 4]]), [(0, 0, [99]), (1, 1, [99])])
    table = p.table_dev.clone()
    table[0, 3] = -1
    p.cache.skv_decode_attn_pages(0, q.cuda(), table, p.lens_dev, lists, i32([[1, 1], [1, 1]]), out)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, 1, 2]), p.table_dev, i32([100, 0]), lists, i32([[1, 1], [1, 1]]), out, 1)
    assert p.cache.skv_get_status() == B.SKV_ERR_BOUNDS


@pytest.mark.parametrize("fp8", [False, True])
def test_nan_reaches_the_result_and_infinities_are_what_they_are(fp8):
    p = Paged([200, 200, 200], 2, 128, fp8=fp8, seed=7)
    q = p.rows(3, 8)
    q[1, 2, 5] = math.nan
    lists, counts = some_lists(random.Random(1), [13] * 3, 2, 6)
    if not fp8:
        bad = torch.randn(1, 2, 128, generator=p.g).bfloat16()
        bad[0, 1, 3] = math.nan
        t = int(lists[2, 1, 0]) * 16
        p.cache.skv_append(0, bad.cuda(), p.v[2][t:t + 1].cuda(), ref.slots_of(p.table, 2, torch.tensor([t])).cuda())
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out)
    nan = torch.isnan(out.cpu()).all(-1)
    want = torch.zeros(3, 8, dtype=torch.bool)
    want[1, 2] = True
    if not fp8:
        want[2, 4:] = True
    assert torch.equal(nan, want) and torch.equal(torch.isnan(out.cpu()).any(-1), want)


# ---- together ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_a_layer_of_prompt_and_steps(hq, hkv, d, fp8):
    """Tables, update, index, selection and attention for a prompt in two chunks and twenty steps, on a layer that owns its
    cache and one that reads it, eagerly and as a captured graph on another stream; with `top` beyond all pages it is
    plain attention."""
    import paper_2604_22782_b200 as skv
    batch, run = 3, 4
    first, second = [70, 33, 5], [30, 0, 44]
    cache = skv.SkvCache([0, 0, 2], hkv, d, 16, 64, allocate=True, fp8=fp8)
    memory, [(codes, scales), (codes2, _)] = index_of(cache, 2)
    g = torch.Generator().manual_seed(d)
    lens, n_free = i32([0] * batch), i32([64])
    table, free = torch.full((batch, 12), -1, dtype=torch.int32, device="cuda"), torch.randperm(64, generator=g).int().cuda()
    k, v = ([torch.zeros(0, hkv, d, dtype=torch.bfloat16) for _ in range(batch)] for _ in range(2))
    have = [0] * batch
    index = {}

    def rows(new):
        x = [torch.randn(sum(new), h, d, generator=g).bfloat16() for h in (hkv, hkv, hq)]
        for b, a in enumerate(new):
            at = slice(sum(new[:b]), sum(new[:b + 1]))
            k[b], v[b] = torch.cat((k[b], x[0][at])), torch.cat((v[b], x[1][at]))
            have[b] += a
        return [y.cuda() for y in x]

    def stored():
        """K, V as the cache holds them."""
        if not fp8:
            return k, v
        t = table.cpu()
        slots = torch.cat([ref.slots_of(t, b, torch.arange(have[b])) for b in range(batch)]).cuda()
        c = [torch.empty(slots.numel(), hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
        s = [torch.empty(slots.numel(), hkv, dtype=torch.float32, device="cuda") for _ in range(2)]
        cache.skv_gather_fp8(0, slots, *c, *s)
        back = [(x.view(torch.float8_e4m3fn).float() * y[..., None]).cpu() for x, y in zip(c, s)]
        return tuple(list(torch.split(x, have)) for x in back)

    class View:
        pass

    def verify(q, out, lists, counts, new, most, this_run, top, first_pages, last_pages):
        p = View()
        p.k, p.v = stored()
        p.lens, p.fp8 = list(have), fp8
        t = table.cpu()
        for b in range(batch):
            for j in range(have[b] // 16):
                for h in range(hkv):
                    c, s = pages.index_entry(p.k[b][16 * j:16 * j + 16, h])
                    at = int(t[b, j])
                    assert torch.equal(codes[at, h].cpu(), c) and float(scales[at, h]) == s
                    index[b, j, h] = c, s
        runs = chunk_runs(have, new, most, this_run)
        group = hq // hkv
        for i, (b, row, pos) in enumerate(runs):
            for h in range(hkv):
                want = []
                if pos:
                    full = have[b] // 16
                    c = torch.stack([index[b, j, h][0] for j in range(full)]) if full else torch.zeros(0, 2, d, dtype=torch.int8)
                    s = torch.tensor([index[b, j, h][1] for j in range(full)])
                    mine = q.cpu()[row:row + len(pos), h * group:(h + 1) * group]
                    want = pages.page_list(pages.scores(mine, c, s) if full else [], pos[0], pos[-1], top, first_pages, last_pages)
                assert lists[i, h, :counts[i, h]].tolist() == want
        check_rows(p, q.cpu(), out, lists.cpu(), counts.cpu(), runs)

    for new in (first, second):
        kk, vv, q = rows(new)
        most = max(new)
        n = sum(new)
        slots, cu = torch.empty(n, dtype=torch.int64, device="cuda"), i32([0] * (batch + 1))
        cache.skv_plan_step(table, lens, i32(new), free, n_free, slots, cu, lens, n_free)
        per = -(-most // run)
        lists = torch.empty(batch * per, hkv, skv.skv_page_list_width(2, 1, 1, run), dtype=torch.int32, device="cuda")
        counts = torch.empty(batch * per, hkv, dtype=torch.int32, device="cuda")
        for layer in (0, 1):
            out = torch.zeros(n, hq, d, dtype=torch.bfloat16, device="cuda")
            cache.skv_append(layer, kk, vv, slots)
            cache.skv_index_pages(layer, table, lens, cu_q_lens=cu, max_q_len=most)
            cache.skv_select_pages(layer, q, table, lens, lists, counts, 2, 1, 1, cu_q_lens=cu, max_q_len=most, run=run)
            cache.skv_prefill_attn_pages(layer, q, cu, table, lens, lists, counts, out, most, run=run)
            verify(q, out, lists, counts, new, most, run, 2, 1, 1)

    ones = i32([1] * batch)
    slots, cu = torch.empty(batch, dtype=torch.int64, device="cuda"), i32([0] * (batch + 1))
    kk, vv, q = (torch.zeros(batch, h, d, dtype=torch.bfloat16, device="cuda") for h in (hkv, hkv, hq))
    out, everything = torch.empty_like(q), torch.empty_like(q)
    lists, all_lists = (torch.empty(batch, hkv, skv.skv_page_list_width(t, 1, 1), dtype=torch.int32, device="cuda") for t in (2, 30))
    counts, all_counts = (torch.empty(batch, hkv, dtype=torch.int32, device="cuda") for _ in range(2))

    def step():
        cache.skv_plan_step(table, lens, ones, free, n_free, slots, cu, lens, n_free)
        cache.skv_append(0, kk, vv, slots)
        cache.skv_index_pages(0, table, lens)
        cache.skv_select_pages(1, q, table, lens, lists, counts, 2)
        cache.skv_decode_attn_pages(1, q, table, lens, lists, counts, out)
        cache.skv_select_pages(0, q, table, lens, all_lists, all_counts, 30)
        cache.skv_decode_attn_pages(0, q, table, lens, all_lists, all_counts, everything)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    plain, ws = torch.empty_like(q), torch.empty(cache.skv_decode_workspace_bytes(batch, hq), dtype=torch.uint8, device="cuda")
    for i in range(20):
        for x, y in zip((kk, vv, q), rows([1] * batch)):
            x.copy_(y)
        if i < 3:
            step()
        else:
            torch.cuda.synchronize()
            if i == 3:
                with torch.cuda.graph(graph, stream=side):           # (capturing runs nothing)
                    step()
            with torch.cuda.stream(side):
                graph.replay()
            side.synchronize()
        torch.cuda.synchronize()
        verify(q, out, lists, counts, [1] * batch, 1, 1, 2, 1, 1)
        cache.skv_decode_attn(0, q, table, lens, plain, ws)
        assert all_counts.tolist() == [[-(-n // 16)] * hkv for n in have]
        p = View()
        p.k, p.v = stored()
        p.lens, p.fp8 = list(have), fp8
        whole = torch.arange(12, dtype=torch.int32).expand(batch, hkv, 12)
        there = torch.tensor([[-(-n // 16)] * hkv for n in have])
        for o in (everything, plain):
            if o is plain and fp8 and d == 128:
                continue                                             # (another arithmetic, with bounds of its own)
            check_rows(p, q.cpu(), o, whole, there, [(b, b, [n - 1]) for b, n in enumerate(have)])
    assert cache.skv_get_status() == 0 and not bool(codes2.any()) and memory.is_cuda


def test_two_streams_at_once():
    """Calls that share nothing but the cache and its index, on two streams."""
    p = Paged([3000] * 4, 2, 128, seed=6)
    _, [(codes, scales)] = index_of(p.cache)
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu_q_lens=i32([0, 3000, 6000, 9000, 12000]), max_q_len=3000)
    q = [p.rows(4, 8).cuda() for _ in range(2)]
    got = [[] for _ in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                lists, counts = torch.empty(4, 2, 40, dtype=torch.int32, device="cuda"), torch.empty(4, 2, dtype=torch.int32, device="cuda")
                out = torch.empty_like(q[i])
                p.cache.skv_select_pages(0, q[i], p.table_dev, p.lens_dev, lists, counts, 30, 1, 8)
                p.cache.skv_decode_attn_pages(0, q[i], p.table_dev, p.lens_dev, lists, counts, out)
                got[i].append((lists, counts, out))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i][1:]:
            assert all(torch.equal(a, b) for a, b in zip(x, got[i][0]))
        lists, counts, out = (x.cpu() for x in got[i][0])
        check_rows(p, q[i].cpu(), out, lists, counts, [(b, b, [2999]) for b in range(4)])
    assert p.cache.skv_get_status() == 0


def test_two_captured_layers_replayed_at_once():
    """No workspace: graphs of the same cache and the same rows may run at the same time."""
    p = Paged([2000, 700], 2, 128, seed=9)
    index_of(p.cache)
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu_q_lens=i32([0, 2000, 2700]), max_q_len=2000)
    q, cu = p.rows(2 * 300, 8).cuda(), i32([0, 300, 600])
    graphs, results, streams = [], [], [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        g = torch.cuda.CUDAGraph()
        lists, counts = torch.empty(2 * 19, 2, 24, dtype=torch.int32, device="cuda"), torch.empty(2 * 19, 2, dtype=torch.int32, device="cuda")
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=s):
            p.cache.skv_select_pages(0, q, p.table_dev, p.lens_dev, lists, counts, 20, cu_q_lens=cu, max_q_len=300, run=16)
            p.cache.skv_prefill_attn_pages(0, q, cu, p.table_dev, p.lens_dev, lists, counts, out, 300, run=16)
        graphs.append(g)
        results.append((lists, counts, out))
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and p.cache.skv_get_status() == 0
    lists, counts, out = (x.cpu() for x in results[0])
    check_rows(p, q.cpu(), out, lists, counts, chunk_runs(p.lens, [300, 300], 300, 16))


def test_both_ways_into_the_library_agree():
    """Plain calls go through the extension; a whole-numbered scale or a given stream through the checked one."""
    p = Paged([500, 90], 2, 128, seed=2)
    index_of(p.cache)
    cu, width = i32([0, 40, 80]), 9
    p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, cu, 500)
    q, one = p.rows(80, 8).cuda(), p.rows(2, 8).cuda()
    got = []
    for scale, stream in ((1.0, None), (1, torch.cuda.current_stream())):
        lists, counts = torch.empty(2 * 5, 2, width, dtype=torch.int32, device="cuda"), torch.empty(2 * 5, 2, dtype=torch.int32, device="cuda")
        few, few_counts = torch.empty(2, 2, width, dtype=torch.int32, device="cuda"), torch.empty(2, 2, dtype=torch.int32, device="cuda")
        out, row = torch.empty_like(q), torch.empty_like(one)
        before = p.cache.skv_launch_count()
        p.cache.skv_index_pages(0, p.table_dev, p.lens_dev, stream=stream)
        p.cache.skv_index_pages(1, p.table_dev, p.lens_dev, stream=stream)       # (not an owner: nothing to do)
        p.cache.skv_select_pages(1, q, p.table_dev, p.lens_dev, lists, counts, 5, 1, 2, cu, 40, 8, stream=stream)
        p.cache.skv_select_pages(1, one, p.table_dev, p.lens_dev, few, few_counts, 5, stream=stream)
        p.cache.skv_prefill_attn_pages(1, q, cu, p.table_dev, p.lens_dev, lists, counts, out, 40, 8, scale, stream=stream)
        p.cache.skv_decode_attn_pages(1, one, p.table_dev, p.lens_dev, few, few_counts, row, scale, stream=stream)
        assert p.cache.skv_launch_count() == before + 5
        got.append((lists, counts, few, few_counts, out, row))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and p.cache.skv_get_status() == 0


def test_refusals():
    import paper_2604_22782_b200 as skv
    from paper_2604_22782_b200.binding import SKV_ERR_ARG, SKV_ERR_LAYER, SKV_ERR_NOMEM, SKV_ERR_UNSUPPORTED, SkvError
    p = Paged([200, 60], 2, 64, seed=1)
    c, table, lens, cu = p.cache, p.table_dev, p.lens_dev, i32([0, 3, 6])
    one, q = p.rows(2, 4).cuda(), p.rows(6, 4).cuda()
    lists, counts = torch.empty(2, 2, 5, dtype=torch.int32, device="cuda"), torch.empty(2, 2, dtype=torch.int32, device="cuda")
    out, rows = torch.empty_like(one), torch.empty_like(q)

    def refused(status, call):
        with pytest.raises(SkvError) as e:
            call()
        assert e.value.status == status

    def select(layer=0, q=one, top=3, first=1, last=1, lists=lists, counts=counts, table=table, **more):
        return lambda: c.skv_select_pages(layer, q, table, lens, lists, counts, top, first, last, **more)

    def decode(layer=0, q=one, out=out, lists=lists, counts=counts):
        return lambda: c.skv_decode_attn_pages(layer, q, table, lens, lists, counts, out)

    def prefill(layer=0, q=q, out=rows, lists=lists, counts=counts, most=3, run=3):
        return lambda: c.skv_prefill_attn_pages(layer, q, cu, table, lens, lists, counts, out, most, run)

    before = c.skv_launch_count()
    refused(SKV_ERR_ARG, lambda: c.skv_index_pages(0, table, lens))                  # no index yet
    refused(SKV_ERR_ARG, select())
    need = c.skv_page_index_bytes()
    memory = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    refused(SKV_ERR_NOMEM, lambda: c.skv_set_page_index(memory[:need - 1]))
    refused(SKV_ERR_ARG, lambda: c.skv_set_page_index(memory[8:]))
    c.skv_set_page_index(memory)
    refused(SKV_ERR_ARG, lambda: c.skv_index_pages(0, table, lens, cu, 0))
    for call in (lambda: c.skv_index_pages(2, table, lens), select(layer=2), select(layer=-1), decode(layer=2), prefill(layer=-1)):
        refused(SKV_ERR_LAYER, call)
    refused(SKV_ERR_ARG, select(top=-1))
    refused(SKV_ERR_ARG, select(first=-1))
    refused(SKV_ERR_ARG, select(last=0))
    refused(SKV_ERR_ARG, select(top=4))                                              # lists of five entries
    refused(SKV_ERR_ARG, select(q=q[:2], max_q_len=3, run=3))                        # rows without offsets
    odd = torch.empty(2 * 4 * 64 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(2, 4, 64)
    three = torch.empty(2, 3, 64, dtype=torch.bfloat16, device="cuda")
    refused(SKV_ERR_ARG, select(q=odd))
    refused(SKV_ERR_ARG, decode(q=odd))
    refused(SKV_ERR_ARG, decode(out=odd))
    refused(SKV_ERR_UNSUPPORTED, select(q=three))
    refused(SKV_ERR_UNSUPPORTED, decode(q=three, out=torch.empty_like(three)))
    refused(SKV_ERR_UNSUPPORTED, prefill(most=65, run=65))                           # 65 rows of two heads
    refused(SKV_ERR_UNSUPPORTED, select(cu_q_lens=cu, max_q_len=65, run=65, lists=torch.empty(2, 2, 9, dtype=torch.int32, device="cuda")))
    long = torch.zeros(2, 45057, dtype=torch.int32, device="cuda")
    refused(SKV_ERR_UNSUPPORTED, select(table=long))
    refused(SKV_ERR_UNSUPPORTED, select(table=long[:, :28673].contiguous(), cu_q_lens=cu, max_q_len=16, run=16, lists=torch.empty(2, 2, 6, dtype=torch.int32, device="cuda")))
    shifted = torch.empty(6 * 4 * 64 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(6, 4, 64)
    c.skv_set_prefill_variant(2)
    refused(SKV_ERR_UNSUPPORTED, prefill(out=shifted))                               # the tile kernel writes 16 bytes at a time
    c.skv_set_prefill_variant(0)
    for call in (select(lists=lists.long()), select(lists=lists[:1]), select(counts=counts[:, :1]), select(q=one.half()), select(q=one[:1]), select(run=0),
                 select(lists=lists.transpose(0, 1)), decode(lists=lists[:, :, ::2]), decode(out=rows), decode(counts=counts.cpu()), decode(q=one[..., :32]),
                 prefill(lists=lists[:1]), prefill(out=out), prefill(run=1), prefill(most=0), prefill(counts=counts.long()),
                 lambda: c.skv_index_pages(0, table[0], lens), lambda: c.skv_index_pages(0, table, lens.long()), lambda: c.skv_index_pages(0, table, lens, cu[:2]),
                 lambda: c.skv_set_page_index(memory.int())):
        with pytest.raises((ValueError, TypeError)):
            call()
    assert c.skv_launch_count() == before and c.skv_get_status() == 0
    c.skv_set_page_index(None)
    refused(SKV_ERR_ARG, select())
    assert skv.skv_page_list_width(3, 1, 1) == 5
