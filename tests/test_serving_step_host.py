"""What of the serving-step operators needs no GPU: descriptions and refusals."""
import math

import pytest
import torch

import paper_2604_22782_b200 as skv
from paper_2604_22782_b200 import binding as B


def test_rope_descriptions_that_are_refused():
    ok = [1.0 / 2 ** i for i in range(32)]
    skv.SkvRope(ok).close()
    skv.SkvRope(ok, axis=[i % 3 for i in range(32)], n_axes=3)

    def refused(status, *a, **kw):
        with pytest.raises(skv.SkvError) as e:
            skv.SkvRope(*a, **kw)
        assert e.value.status == status

    refused(B.SKV_ERR_ARG, [])
    refused(B.SKV_ERR_UNSUPPORTED, ok[:7])                      # 14 dims: not a multiple of 16
    refused(B.SKV_ERR_UNSUPPORTED, [1.0] * 72)                  # 144 dims
    refused(B.SKV_ERR_ARG, ok, n_axes=0)
    refused(B.SKV_ERR_UNSUPPORTED, ok, n_axes=300)
    refused(B.SKV_ERR_ARG, ok, axis=[3] * 32, n_axes=3)
    refused(B.SKV_ERR_ARG, ok, axis=[-1] * 32, n_axes=3)
    for x in (math.nan, math.inf, -math.inf, 1e7):
        refused(B.SKV_ERR_ARG, ok[:-1] + [x])
    with pytest.raises(ValueError):
        skv.SkvRope(ok, axis=[0])


def test_a_handle_without_memory_launches_nothing():
    c = skv.SkvCache([0, 0], 2, 64, 16, 4, accounting_only=True)
    rope = skv.SkvRope([1.0] * 32)
    a = B.SKV_ERR_ARG
    assert B.lib.skv_rope_append(c._h, 0, rope._h, None, 0, None, 0, None, 0, None, 0, None, 0, None, 1, 0, None) == a
    assert B.lib.skv_plan_step(c._h, None, 1, None, None, 1, None, 0, None, 0, None, None, None, None, None, None) == a
    assert B.lib.skv_plan_release(c._h, None, 1, None, None, 1, None, 0, None, None, None) == a
    assert B.lib.skv_decode_attn_window(c._h, 0, None, None, None, None, 1, 2, 1, 1, 0, 0.0, None, 0, None) == a
    assert B.lib.skv_prefill_attn_window(c._h, 0, None, None, None, None, None, 1, 1, 2, 1, 1, 0, 0.0, None) == a
    assert B.lib.skv_rope_append(None, 0, rope._h, None, 0, None, 0, None, 0, None, 0, None, 0, None, 1, 0, None) == a
    assert c.skv_launch_count() == 0


def test_host_tensors_are_refused():
    c = skv.SkvCache([0], 2, 64, 16, 4, accounting_only=True)
    q, i = torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        c.skv_decode_attn_window(0, q, i[None], i, q, torch.zeros(1, dtype=torch.uint8), 4)
    with pytest.raises(ValueError):
        c.skv_prefill_attn_window(0, q, torch.zeros(2, dtype=torch.int32), i[None], i, q, 1, 4)
    with pytest.raises(ValueError):
        c.skv_rope_append(0, skv.SkvRope([1.0] * 32), q, q, q, q, i, i.long())
    with pytest.raises(ValueError):
        c.skv_plan_step(i[None], i, i, i, i, i.long(), torch.zeros(2, dtype=torch.int32), i, i)


def test_the_reference_agrees_with_itself():
    """The plain statements against brute force: the window's mask, and a plan of one page."""
    n, window, sinks = 9, 3, 2
    q, k = torch.zeros(n, 1, 4), torch.zeros(n, 1, 4)
    import serving_reference as ref
    v = torch.eye(n).repeat_interleave(1, 0)[:, None, :]
    out, _, _ = ref.attention(q.repeat(1, 1, 1), k, torch.nn.functional.pad(v, (0, 0))[:, :, :4], torch.arange(n), window, sinks)
    for pos in range(n):
        seen = [t for t in range(n) if ref.sees(pos, t, window, sinks)]
        assert torch.allclose(out[pos, 0], torch.tensor([1.0 / len(seen) if t in seen else 0.0 for t in range(4)], dtype=torch.float64))
    assert ref.plan_step([[7, -1]], [16], [2], [3, 4], 2, 9) == ([[7, 4]], [64, 65], [16, 17], [0, 2], [18], 1, [])
