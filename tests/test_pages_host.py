"""What of the selected-pages operators needs no GPU: sizes and refusals, and the plain statements against brute force."""
import math

import pytest
import torch

import pages_reference as pages
import paper_2604_22782_b200 as skv
from paper_2604_22782_b200 import binding as B

NAMES = ["index_pages", "select_pages", "decode_attn_pages", "prefill_attn_pages"]


def test_sizes():
    for r, hkv, d, n in (([0], 1, 64, 1), ([0, 0, 2, 2], 8, 128, 1000), ([0, 1, 2], 3, 64, 77)):
        c = skv.SkvCache(r, hkv, d, 16, n, accounting_only=True)
        up = lambda x: -(-x // 256) * 256  # noqa: E731
        assert c.skv_page_index_bytes() == len(set(r)) * (up(n * hkv * 2 * d) + up(n * hkv * 4))
    assert skv.skv_page_list_width(10, 1, 2) == 13 and skv.skv_page_list_width(10, 1, 2, 2) == 14
    assert skv.skv_page_list_width(0, 0, 1, 17) == 2 and skv.skv_page_list_width(0, 0, 1, 18) == 3
    assert skv.skv_page_list_width(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1) == 2 ** 31 - 1
    for bad in ((-1, 0, 1, 1), (0, -1, 1, 1), (0, 0, 0, 1), (0, 0, 1, 0)):
        with pytest.raises(skv.SkvError):
            skv.skv_page_list_width(*bad)
    with pytest.raises(ValueError):
        skv.skv_page_list_width(1 << 40, 0, 1)


def test_width_is_enough_for_every_run():
    for run in (1, 2, 5, 16, 17, 32, 128):
        for p0 in range(40):
            got = pages.page_list([0.0] * 100, p0 + 800, p0 + 800 + run - 1, 7, 2, 3)
            assert len(got) <= skv.skv_page_list_width(7, 2, 3, run) and got == sorted(set(got))


def test_a_handle_without_memory_launches_nothing():
    c = skv.SkvCache([0, 0], 2, 64, 16, 4, accounting_only=True)
    a = B.SKV_ERR_ARG
    assert B.lib.skv_index_pages(c._h, 0, None, None, None, 1, 1, 1, None) == a
    assert B.lib.skv_select_pages(c._h, 0, None, None, None, None, None, None, 1, 1, 2, 1, 1, 1, 1, 1, 3, None) == a
    assert B.lib.skv_decode_attn_pages(c._h, 0, None, None, None, None, None, None, 1, 2, 1, 1, 0.0, None) == a
    assert B.lib.skv_prefill_attn_pages(c._h, 0, None, None, None, None, None, None, None, 1, 1, 2, 1, 1, 1, 0.0, None) == a
    assert B.lib.skv_set_page_index(c._h, 256, 1 << 20, None) == a and B.lib.skv_set_page_index(None, None, 0, None) == a
    assert B.lib.skv_set_page_index(c._h, None, 0, None) == 0
    assert B.lib.skv_page_index_bytes(c._h, None) == a and c.skv_launch_count() == 0


def test_host_tensors_are_refused():
    c = skv.SkvCache([0], 2, 64, 16, 4, accounting_only=True)
    q, i = torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    lists, counts, cu = torch.zeros(1, 2, 3, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: c.skv_set_page_index(torch.zeros(1 << 16, dtype=torch.uint8)), lambda: c.skv_index_pages(0, i[None], i),
                 lambda: c.skv_select_pages(0, q, i[None], i, lists, counts, 1), lambda: c.skv_decode_attn_pages(0, q, i[None], i, lists, counts, q),
                 lambda: c.skv_prefill_attn_pages(0, q, cu, i[None], i, lists, counts, q, 1)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("name", NAMES)
def test_the_extension_declines_what_is_not_plain(name):
    f = getattr(B._calls, name)
    host = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for args in ((), (None,), (1,), (0, host), (1 << 70, host), (-1, host), ("x", "y"), (1, host), (1, None) + (3,) * 12, (1, host) + (host,) * 11,
                 (1, host) + (None,) * 11, (1, host) + (1,) * 40):
        assert f(*args) is None
    for args in ((), (1, 2, 3), (0, 1, 2, 3), ("a",) * 4):
        with pytest.raises((TypeError, ValueError)):
            B._calls.connect_pages(*args)


def test_the_reference_agrees_with_itself():
    """The score is the largest over a page's box of bounds; attention with everything listed is softmax attention; ties."""
    g = torch.Generator().manual_seed(0)
    k = torch.randn(16, 4, generator=g)
    codes, scale = pages.index_entry(k)
    q = torch.randn(1, 1, 4, generator=g)
    best = max(sum(float(c) * int(codes[(m >> i) & 1, i]) for i, c in enumerate(pages.steps(q.numpy(), q.abs().max().item())[0, 0])) for m in range(16))
    assert float(pages.scores(q, codes[None], torch.tensor([scale]))[0]) == float(torch.tensor(best).float() * torch.tensor(scale).float())
    assert pages.index_entry(torch.full((16, 4), math.nan))[1] == math.inf
    assert pages.page_list([1.0, 5.0, 5.0, 5.0, 0.0], 79, 79, 2, 0, 1) == [1, 2, 4]
    n = 20
    k, v, q = (torch.randn(n, 4, generator=g) for _ in range(3))
    out, _, _ = pages.attention(q[:, None], k, v, torch.arange(n), [1, 0])
    x = (q.double() @ k.double().T / 2).masked_fill(torch.triu(torch.ones(n, n, dtype=torch.bool), 1), -math.inf)
    assert torch.allclose(out[:, 0], torch.softmax(x, 1) @ v.double())
