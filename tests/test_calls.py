"""The marshalling extension of the serving step's calls: what it declines goes through the checks written in Python."""
import ctypes

import pytest
import torch

import paper_2604_22782_b200 as skv
from paper_2604_22782_b200 import binding
from paper_2604_22782_b200.binding import SkvError, _calls

NAMES = ["decode_attn_window", "prefill_attn_window", "rope_append", "plan_step", "plan_release"]


@pytest.mark.parametrize("name", NAMES)
def test_anything_that_is_not_plain_is_declined(name):
    f = getattr(_calls, name)
    host = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for args in ((), (None,), (1,), (0, host), (1 << 70, host), (-1, host), ("x", "y"), (1, host), (1, None) + (3,) * 12, (1, host) + (host,) * 11,
                 (1, host) + (None,) * 11, (1, host) + (1,) * 40):
        assert f(*args) is None


def test_connect_refuses_what_is_no_address():
    for args in ((), (1, 2, 3), (0, 1, 2, 3, 4, 5), ("a",) * 6):
        with pytest.raises((TypeError, ValueError)):
            _calls.connect(*args)
    entry = [binding.lib.skv_is_owner, binding.lib.skv_rope_append, binding.lib.skv_plan_step, binding.lib.skv_plan_release,
             binding.lib.skv_decode_attn_window, binding.lib.skv_prefill_attn_window]
    _calls.connect(*(ctypes.cast(f, ctypes.c_void_p).value for f in entry))          # (as it was)


def test_closed_handles_are_refused():
    cache = skv.SkvCache([0], 2, 64, 16, 4, accounting_only=True)
    rope = skv.SkvRope([0.5] * 32)
    rope.close()
    cache.close()
    assert cache._handle is None and rope._handle is None
    with pytest.raises((SkvError, ValueError)):
        cache.skv_plan_release(torch.zeros(1, 1, dtype=torch.int32), *(torch.zeros(1, dtype=torch.int32) for _ in range(5)))


@pytest.mark.gpu
def test_plain_calls_take_it_and_others_give_the_same():
    """The same arguments with an integer scale or a stream given are not plain: both ways, one result."""
    cache = skv.SkvCache([0, 0], 2, 64, 16, 8, allocate=True)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(40, 2, 64, generator=g).bfloat16().cuda() for _ in range(2))
    q = torch.randn(40, 4, 64, generator=g).bfloat16().cuda()
    slots = torch.arange(40, device="cuda")
    rope, pos = skv.SkvRope([1.0 / (1 + i) for i in range(32)]), torch.arange(40, dtype=torch.int32, device="cuda")
    table, lens = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([40], dtype=torch.int32, device="cuda")
    ws = torch.empty(cache.skv_decode_workspace_bytes(1, 4), dtype=torch.uint8, device="cuda")
    cu = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    s = torch.cuda.current_stream()
    turned = [torch.empty_like(q) for _ in range(3)]
    head = (cache._handle, cache.pool)
    assert _calls.rope_append(*head, 64, 2, 1, 0, rope._handle, q, turned[0], k, v, pos, slots, None) == 0
    cache.skv_rope_append(0, rope, q, turned[1], k, v, pos, slots)
    cache.skv_rope_append(0, rope, q, turned[2], k, v, pos, slots, stream=s)
    assert _calls.rope_append(*head, 64, 2, 1, 1, rope._handle, q, turned[0], None, None, pos, None, None) == 0      # layer 1 keeps nothing
    assert all(torch.equal(t, turned[0]) for t in turned)
    assert _calls.rope_append(*head, 64, 2, 1, 0, rope._handle, q, turned[0], k, v, pos, slots, s) is None
    one = [torch.empty(1, 4, 64, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    assert _calls.decode_attn_window(*head, 64, 1, q[:1], table, lens, one[0], ws, 20, 3, 0.25, None) == 0
    cache.skv_decode_attn_window(1, q[:1], table, lens, one[1], ws, 20, 3, scale=0.25)
    cache.skv_decode_attn_window(1, q[:1], table, lens, one[2], ws, 20, 3, scale=0.25, stream=s)
    assert all(torch.equal(o, one[0]) for o in one)
    rows = [torch.empty_like(q) for _ in range(3)]
    assert _calls.prefill_attn_window(*head, 64, 1, q, cu, table, lens, rows[0], 40, 20, 3, 1.0, None) == 0
    cache.skv_prefill_attn_window(1, q, cu, table, lens, rows[1], 40, 20, 3, scale=1.0)
    cache.skv_prefill_attn_window(1, q, cu, table, lens, rows[2], 40, 20, 3, scale=1, stream=s)
    assert all(torch.equal(o, rows[0]) for o in rows)
    with pytest.raises(SkvError):
        cache.skv_decode_attn_window(5, q[:1], table, lens, one[0], ws, 20, 3)
    for bad in ((q[:1].float(), lens), (q[:1], lens.long()), (q[:1], lens.cpu()), (q[0], lens), (q[:2], lens)):
        with pytest.raises((TypeError, ValueError)):
            cache.skv_decode_attn_window(1, bad[0], table, bad[1], one[0], ws, 20, 3)
    assert cache.skv_get_status() == 0
