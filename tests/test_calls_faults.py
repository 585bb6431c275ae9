"""Arguments whose inspection throws: the marshalling extension declines them, and the call raises.  In
processes of their own, which an exception that nobody catches would end."""
import subprocess
import sys
import textwrap

import pytest

PREPARE = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_2604_22782_b200 as skv
from paper_2604_22782_b200 import binding
with FakeTensorMode():
    def fake(*shape, dtype=torch.int32):
        return torch.empty(*shape, dtype=dtype, device="cuda:0")
    q, table, lens, ws = fake(2, 4, 64, dtype=torch.bfloat16), fake(2, 3), fake(2), fake(1 << 20, dtype=torch.uint8)
    k, cu, slots, one, pages, pool = fake(2, 2, 64, dtype=torch.bfloat16), fake(3), fake(2, dtype=torch.int64), fake(1), fake(9), fake(1 << 20, dtype=torch.uint8)
def refused(status):                  # declined, or the entry point's own refusal of a null pointer, where asking for one does not throw
    return status is None or status < 0
cache, rope = skv.SkvCache([0], 2, 64, 16, 4, accounting_only=True), skv.SkvRope([0.5] * 32)
ARGS = dict(
    decode_attn_window=(64, 0, q, table, lens, q, ws, 8, 0, 0.0, None),
    prefill_attn_window=(64, 0, q, cu, table, lens, q, 2, 8, 0, 0.0, None),
    rope_append=(64, 2, 1, 0, rope._handle, q, q, k, k, lens, slots, None),
    plan_step=(table, lens, lens, pages, one, slots, cu, lens, one, None, None),
    plan_release=(table, lens, lens, pages, one, one, None),
)
CALLS = dict(
    decode_attn_window=lambda c: c.skv_decode_attn_window(0, q, table, lens, q, ws, 8, 0),
    prefill_attn_window=lambda c: c.skv_prefill_attn_window(0, q, cu, table, lens, q, 2, 8, 0),
    rope_append=lambda c: c.skv_rope_append(0, rope, q, q, k, k, lens, slots),
    plan_step=lambda c: c.skv_plan_step(table, lens, lens, pages, one, slots, cu, lens, one),
    plan_release=lambda c: c.skv_plan_release(table, lens, lens, pages, one, one),
)
"""


def run(code):
    r = subprocess.run([sys.executable, "-c", PREPARE + textwrap.dedent(code)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, f"{r.returncode}: {r.stdout} {r.stderr[-500:]}"


def test_a_pool_without_memory_is_refused_and_the_call_raises():
    """(Without a device the question for the current one throws; with one, the tensors' pointers may.)"""
    run("""
    for name in ARGS:
        print(name, flush=True)
        assert refused(getattr(binding._calls, name)(cache._handle, pool, *ARGS[name]))
    cache.pool = pool
    for name in CALLS:
        try:
            CALLS[name](cache)
        except Exception:
            continue
        raise SystemExit(f"{name}: nothing was raised")
    """)


@pytest.mark.gpu
def test_tensors_without_memory_beside_a_real_pool():
    run("""
    cache = skv.SkvCache([0], 2, 64, 16, 4, allocate=True)
    before = cache.skv_launch_count()
    for name in ARGS:
        print(name, flush=True)
        assert refused(getattr(binding._calls, name)(cache._handle, cache.pool, *ARGS[name]))
        try:
            CALLS[name](cache)
        except Exception:
            continue
        raise SystemExit(f"{name}: nothing was raised")
    assert cache.skv_launch_count() == before and cache.skv_get_status() == 0
    """)
