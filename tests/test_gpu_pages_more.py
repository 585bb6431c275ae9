"""Attention over selected pages once more: caches of many rounds of scores and of the widest tables, FP8 values of every size, FP8
pages that hold anything where nobody looks."""
import math
import random

import pytest
import torch

import pages_reference as pages
import serving_reference as ref
from test_gpu_pages import Indexed, check, check_rows, chunk_runs, i32
from test_gpu_window import Paged

pytestmark = pytest.mark.gpu


# ---- the selection -------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("kind", ["drawn", "ties", "equal", "wild"])
@pytest.mark.parametrize("batch", [1, 3, 40])
def test_selection_over_several_rounds_of_scores(batch, kind):
    """Up to 2500 pages, 2048 of them to a round, of few different scores, of one alone, of many infinite ones; `top` on both sides
    of a round."""
    lens = [40000 - 211 * b for b in range(batch)]
    p = Indexed(lens, 2, 64, seed=batch, kind=kind)
    q = torch.randn(batch, 4, 64, generator=p.g).bfloat16()
    for top, first, last in ((100, 1, 8), (2047, 0, 1), (2048, 3, 2), (2049, 1, 1), (2300, 0, 5)):
        lists, counts = p.select(q, top, first, last)
        p.check(q, lists, counts, top, first, last)
    if batch == 3:                                            # runs: few columns and many
        new = [20, 9, 31]
        q = torch.randn(sum(new), 4, 64, generator=p.g).bfloat16()
        for run in (4, 31):
            for top in (300, 2048, 2060):
                lists, counts = p.select(q, top, 2, 3, new, 31, run)
                p.check(q, lists, counts, top, 2, 3, new, 31, run)


@pytest.mark.parametrize("kind", ["drawn", "ties", "wild"])
@pytest.mark.parametrize("width,run", [(45056, 1), (45056, 8), (28672, 64), (28672, 9)])
def test_selection_in_the_longest_caches(width, run, kind):
    """Tables as wide as they may be, two query heads a kv head: up to 16 columns, and more."""
    n, new = 16 * width - 5, 64
    p = Indexed([n], 2, 64, seed=width + run, kind=kind)
    assert p.table.shape[1] == width
    q = torch.randn(new, 4, 64, generator=p.g).bfloat16()
    for top, first, last in ((100, 1, 8), (20000, 0, 1)):
        if run == 1:
            lists, counts = p.select(q[:1], top, first, last)
            p.check(q[:1], lists, counts, top, first, last)
        else:
            lists, counts = p.select(q, top, first, last, [new], new, run)
            p.check(q, lists, counts, top, first, last, [new], new, run)


# ---- attention on FP8 pages ----------------------------------------------------------------------------------------
def stored(p):
    """K, V of every sequence as the FP8 cache holds them."""
    slots = torch.cat([ref.slots_of(p.table, b, torch.arange(n)) for b, n in enumerate(p.lens)]).cuda()
    hkv, d = p.cache.kv_heads, p.cache.head_dim
    codes = [torch.empty(slots.numel(), hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty(slots.numel(), hkv, dtype=torch.float32, device="cuda") for _ in range(2)]
    p.cache.skv_gather_fp8(0, slots, *codes, *scales)
    back = [(c.view(torch.float8_e4m3fn).double() * s.double()[..., None]).cpu() for c, s in zip(codes, scales)]
    return [list(torch.split(x, p.lens)) for x in back]


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("far", [-85, 0, 60, 100, 107])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_fp8_values_of_every_size(hq, hkv, d, far, variant):
    """4095 tokens of a 4096th of the weight each, beside one that has as much as all of them and V = 0: their sum has to be there whatever V's
    size, from 2^-91 to what 4096 times it stays below 2^120."""
    n, a, run = 4096, 8, 8
    p = Paged([n], hkv, d, True, seed=d)
    p.cache.skv_set_prefill_variant(variant)
    q = torch.zeros(a, hq, d)
    q[..., 0] = 4.0
    k = torch.zeros(n, hkv, d)
    k[5, :, 0] = 12 * math.log(2) * math.sqrt(d) / 4.0       # 2^12 times the weight of each of the others
    v = torch.rand(n, hkv, d, generator=p.g) + 0.5
    v[5] = 0.0
    v *= 2.0 ** far
    slots = ref.slots_of(p.table, 0, torch.arange(n)).cuda()
    p.cache.skv_append(0, k.bfloat16().cuda(), v.bfloat16().cuda(), slots)
    p.k, p.v = stored(p)
    q = q.bfloat16()
    runs = chunk_runs([n], [a], a, run)
    lists = torch.arange(n // 16, dtype=torch.int32).expand(1, hkv, -1).contiguous()
    counts = torch.full((1, hkv), n // 16, dtype=torch.int32)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, a]), p.table_dev, p.lens_dev, lists.cuda(), counts.cuda(), out, a, run=run)
    # A probability times V scale over c is 2^-13.6 or more (V within a factor of three), a normal number of f16: 2^-11 of it, and
    # nothing for the smallest steps.
    for i, (b, row, pos) in enumerate(runs):
        for h in range(hkv):
            mine = slice(row, row + len(pos)), slice(h * hq // hkv, (h + 1) * hq // hkv)
            want = pages.attention(q[mine], p.k[b][:, h], p.v[b][:, h], torch.tensor(pos), lists[i, h].tolist())
            check(out[mine], want + (n, True, 0.0), f"2^{far} head {h}")
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("byte", [0x7F, 0xFF, 0x00])
@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64), (4, 4, 128)])
def test_fp8_pages_and_slots_that_nobody_sees_may_hold_anything(hq, hkv, d, variant, byte):
    """Pages that are not listed and, in those that are, slots behind the sequence's end: NaN codes, scales of NaN or far out."""
    lens, new = [1000, 333], [20, 7]
    p = Paged(lens, hkv, d, True, seed=d)
    p.cache.skv_set_prefill_variant(variant)
    q = p.rows(27, hq)
    runs = chunk_runs(lens, new, 20, 4)
    rng = random.Random(d)
    some = [sorted(rng.sample(range(n // 16 - 2), 9)) for n in lens]
    lists = torch.full((len(runs), hkv, 12), -1, dtype=torch.int32)
    counts = torch.zeros((len(runs), hkv), dtype=torch.int32)
    for i, (b, _, pos) in enumerate(runs):
        if pos:
            mine = some[b] + list(range(pos[0] // 16, pos[-1] // 16 + 1))
            lists[i, :, :len(mine)], counts[i] = torch.tensor(mine, dtype=torch.int32), len(mine)
    table = p.table.clone()
    block = 32 * (d + 4)
    body = p.cache.pool[256:].view(-1, hkv, block)
    held_pages = set()
    for b, n in enumerate(lens):
        held = set(some[b]) | set(range((n - new[b]) // 16, -(-n // 16)))
        held_pages |= {int(p.table[b, j]) for j in held}
        for j in range(-(-n // 16)):
            if j not in held:
                table[b, j] = -1 if j % 2 else 1 << 30
        last, used = int(p.table[b, (n - 1) // 16]), (n - 1) % 16 + 1
        k = body[last, :, :16 * d].view(hkv, 2, d // 16, 8, 16)
        v = body[last, :, 16 * d:32 * d].view(hkv, d, 16)
        s = body[last, :, 32 * d:].view(hkv, 2, 16, 4)
        for t in range(used, 16):
            k[:, t // 8, :, t % 8], v[:, :, t], s[:, :, t] = byte, byte, byte
    body[[j for j in range(body.shape[0]) if j not in held_pages]] = byte
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_prefill_attn_pages(0, q.cuda(), i32([0, 20, 27]), table.cuda(), p.lens_dev, lists.cuda(), counts.cuda(), out, 20, run=4)
    check_rows(p, q, out, lists, counts, runs)
    ends = [19, 26]
    one = torch.empty(2, hq, d, dtype=torch.bfloat16, device="cuda")
    own = [max(i for i, r in enumerate(runs) if r[0] == b and r[2]) for b in range(2)]
    p.cache.skv_decode_attn_pages(0, q[ends].cuda(), table.cuda(), p.lens_dev, lists[own].contiguous().cuda(), counts[own].contiguous().cuda(), one)
    check_rows(p, q[ends], one, lists[own], counts[own], [(b, b, [lens[b] - 1]) for b in range(2)])
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_attention_far_into_a_long_table(fp8):
    """Pages all over the widest table that a selection takes, the last one partly filled."""
    width, hkv, d, hq = 45056, 2, 64, 6
    n = 16 * width - 3
    held = sorted(random.Random(1).sample(range(width), 300) + [width - 1])
    p = Paged([16 * len(held)], hkv, d, fp8, seed=5)
    table = torch.full((1, width), -1, dtype=torch.int32)
    table[0, held] = p.table[0, :len(held)]
    k, v = (torch.zeros(n + 3, hkv, d, dtype=torch.float64) for _ in range(2))
    at = torch.tensor([16 * j + t for j in held for t in range(16)])
    k[at], v[at] = p.k[0].double(), p.v[0].double()
    p.k, p.v, p.lens = [k[:n]], [v[:n]], [n]
    lists = torch.tensor(held, dtype=torch.int32).expand(1, hkv, -1).contiguous()
    counts = torch.full((1, hkv), len(held), dtype=torch.int32)
    q = p.rows(1, hq)
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    p.cache.skv_decode_attn_pages(0, q.cuda(), table.cuda(), i32([n]), lists.cuda(), counts.cuda(), out)
    check_rows(p, q, out, lists, counts, [(0, 0, [n - 1])])
    rows = p.rows(20, hq)
    for variant in (1, 2):
        p.cache.skv_set_prefill_variant(variant)
        out = torch.empty(rows.shape, dtype=torch.bfloat16, device="cuda")
        p.cache.skv_prefill_attn_pages(0, rows.cuda(), i32([0, 20]), table.cuda(), i32([n]), lists.cuda(), counts.cuda(), out, 20, run=20)
        check_rows(p, rows, out, lists, counts, [(0, 0, list(range(n - 20, n)))])
    assert p.cache.skv_get_status() == 0
