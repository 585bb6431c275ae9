"""Values that some rows of a chunk see and others must not: at bf16's largest and lowest, a weight that is not exactly zero
would show in the rows that do not see them."""
import pytest
import torch

import serving_reference as ref
from test_gpu_window import Paged, chunk

pytestmark = pytest.mark.gpu

LENS = [700, 300, 90]


def extreme(p, value):
    """Some tokens of every sequence, at all places of a page among them, get this value in every dim."""
    marked = []
    for b, n in enumerate(p.lens):
        t = torch.tensor([x for x in range(30, n, 17) if x // 17 % 9 == 0] + [46, 47, 62, 63, n - 30, n - 29])
        t = t.unique()
        rows = torch.full((len(t),) + p.v[b].shape[1:], value, dtype=torch.bfloat16)
        p.cache.skv_append(0, p.k[b][t].bfloat16().cuda(), rows.cuda(), ref.slots_of(p.table, b, t).cuda())
        p.v[b][t] = rows.to(p.v[b].dtype)
        marked.append(t)
    return marked


@pytest.mark.parametrize("value", [torch.finfo(torch.bfloat16).min, torch.finfo(torch.bfloat16).max])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 64)])
@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("window,sinks", [(20, 0), (100, 4), (5000, 0)])
def test_rows_that_do_not_see_an_extreme_value(window, sinks, variant, hq, hkv, d, value):
    p = Paged(LENS, hkv, d, seed=61)
    p.cache.skv_set_prefill_variant(variant)
    hold(p, hq, window, sinks, value)


def hold(p, hq, window, sinks, value, more=lambda size, reach: 0.0):
    marked = extreme(p, value)
    q = p.rows(sum(LENS), hq)
    out = chunk(p, q, LENS, window, sinks).double().cpu()
    at = compared = 0
    for b, n in enumerate(LENS):
        pos, t = torch.arange(n), marked[b]
        seen = (t[None] <= pos[:, None]) & ((t[None] > pos[:, None] - window) | (t[None] < sinks))
        clear = ~seen.any(1)
        plain = p.v[b].clone()
        plain[t] = 0.0                                    # (what the clear rows are to get does not depend on them)
        want, size, reach = ref.attention(q[at:at + n], p.k[b], plain, pos, window, sinks)
        tol = ref.attention_tolerance(want, size, reach, n, p.fp8, float(plain.double().abs().max())) + more(size, reach)
        bad = ((out[at:at + n] - want).abs() <= tol).logical_not()[clear]
        assert not bool(bad.any()), f"length {n}: {int(bad.sum())} of {bad.numel()}"
        compared += int(clear.sum())
        at += n
    assert compared >= 100
    assert p.cache.skv_get_status() == 0


@pytest.mark.parametrize("value", [torch.finfo(torch.bfloat16).min, torch.finfo(torch.bfloat16).max])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 128), (6, 2, 64)])
@pytest.mark.parametrize("scratch", [False, True])
@pytest.mark.parametrize("window,sinks", [(20, 0), (100, 4), (5000, 0)])
def test_rows_on_fp8_pages_that_do_not_see_an_extreme_value(window, sinks, scratch, hq, hkv, d, value):
    """By the kernel that reads the codes, and through a scratch area (K, V rounded to bf16 there: 2^-8 of themselves, which moves
    a score by 2^-8 of the row's reach, and a weight and the weights' sum by as much)."""
    p = Paged(LENS, hkv, d, fp8=True, seed=62)
    if not scratch:
        return hold(p, hq, window, sinks, value)
    p.cache.skv_set_prefill_scratch(torch.empty(p.cache.skv_prefill_scratch_bytes(), dtype=torch.uint8, device="cuda"))
    hold(p, hq, window, sinks, value, lambda size, reach: size * (2 ** -8 + 2 * 2 ** -8 * reach) + size * 2 ** -8)
    p.cache.skv_set_prefill_scratch(None)
