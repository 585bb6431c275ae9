"""Rotary embedding with the update against a 64-bit statement of it: pair layouts, position axes, partial rotation, far and
negative positions, strided rows, any slot map, FP8 pages, layers that keep nothing."""
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu

HEADS = [(8, 2, 128), (32, 8, 128), (4, 4, 128), (6, 2, 64), (1, 1, 64), (3, 3, 128)]


def freqs(rotary, theta=1e6):
    return [theta ** (-2.0 * i / rotary) for i in range(rotary // 2)]


def inputs(n, hq, hkv, d, g, fused):
    """Rows of their own, or slices of a fused projection's."""
    if fused:
        rows = torch.randn(n, (hq + 2 * hkv) * d, generator=g).bfloat16()
        dev = rows.cuda()
        cut = lambda x: (x[:, :hq * d].view(n, hq, d), x[:, hq * d:(hq + hkv) * d].view(n, hkv, d), x[:, (hq + hkv) * d:].view(n, hkv, d))  # noqa: E731
        return cut(rows), cut(dev)
    host = tuple(torch.randn(n, h, d, generator=g).bfloat16() for h in (hq, hkv, hkv))
    return host, tuple(x.cuda() for x in host)


def check_rows(got, x, angle, adjacent, what):
    want, size = ref.rope(x, angle, adjacent)
    err, tol = (got.double().cpu() - want).abs(), ref.rope_tolerance(want, size)
    assert bool((err <= tol).all()), f"{what}: {(err - tol).max().item()}"


def run(n, hq, hkv, d, rotary, axes, adjacent, fp8, positions, slots, pages, g, fused=True, r=(0, 0), layer=0):
    import paper_2604_22782_b200 as skv
    axis = [i % axes for i in range(rotary // 2)]
    rope = skv.SkvRope(freqs(rotary), axis=axis, n_axes=axes, adjacent_pairs=adjacent)
    cache = skv.SkvCache(list(r), hkv, d, 16, pages, allocate=True, fp8=fp8)
    (q, k, v), (qd, kd, vd) = inputs(n, hq, hkv, d, g, fused)
    out = torch.full((n, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    cache.skv_rope_append(layer, rope, qd, out, kd, vd, positions.cuda(), slots.cuda())
    torch.cuda.synchronize()
    angle = ref.angles(positions.view(axes, n), freqs(rotary), axis)
    check_rows(out, q, angle, adjacent, "queries")
    assert torch.equal(qd.cpu(), q) and torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)      # inputs left as they were
    return cache, (q, k, v), angle


def check_stored(cache, k, v, slots, angle, adjacent, fp8):
    n, hkv, d = k.shape
    live = slots >= 0
    ids = slots[live].cuda()
    m = ids.numel()
    if not fp8:
        ko, vo = (torch.empty(m, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache.skv_gather(0, ids, ko, vo)
        check_rows(ko, k[live], angle[live], adjacent, "keys")
        assert torch.equal(vo.cpu(), v[live])
        return
    kc, vc = (torch.empty(m, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.empty(m, hkv, device="cuda") for _ in range(2))
    cache.skv_gather_fp8(0, ids, kc, vc, ks, vs)
    for codes, scales, want, size in ((kc, ks, *ref.rope(k[live], angle[live], adjacent)), (vc, vs, v[live].double(), torch.zeros(m, hkv, d))):
        top = want.abs().amax(-1)
        scales, codes = scales.cpu().double(), codes.view(torch.float8_e4m3fn).double().cpu()
        # the scale: the row's maximum (off as an fp32 rotation is) and one division
        assert bool(((scales - top / 448).abs() <= top / 448 * 2 ** -23 + size.amax(-1) / 448 * 2 ** -20).all())
        # a code is half a step off (2^-4 of it, or half of the smallest step 2^-9), beside the rotation's and two products' errors
        err = (codes * scales[..., None] - want).abs()
        assert bool((err <= want.abs() * (2 ** -4 + 2 ** -20) + scales[..., None] * 2 ** -10 + size * 2 ** -19).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_head_shapes_and_axes(hq, hkv, d, adjacent, fp8):
    g = torch.Generator().manual_seed(hq * 7 + d)
    for n, rotary, axes in ((1, d, 1), (7, d, 3), (33, d // 2, 1), (300, d, 3), (50, 16, 4), (1001, d, 1)):
        pages = n // 16 + 3
        slots = torch.randperm(pages * 16, generator=g)[:n]
        positions = torch.randint(0, 40000, (axes, n), generator=g, dtype=torch.int32)
        cache, (q, k, v), angle = run(n, hq, hkv, d, rotary, axes, adjacent, fp8, positions, slots, pages, g, fused=n % 2 == 1)
        check_stored(cache, k, v, slots, angle, adjacent, fp8)
        assert cache.skv_get_status() == 0


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (6, 2, 64)])
def test_whole_pages_in_order_holes_and_ragged_ends(hq, hkv, d, fp8):
    """What a prompt's slots look like: whole pages in a random order, one starting inside a page, one with holes."""
    g = torch.Generator().manual_seed(5)
    n, pages = 700, 60
    order = torch.randperm(pages, generator=g)
    t = torch.arange(n)
    for shift, holes in ((0, False), (5, False), (0, True), (13, True)):
        slots = order[(t + shift) // 16] * 16 + (t + shift) % 16
        if holes:
            slots[torch.randint(0, n, (90,), generator=g)] = -1
        positions = (t + 100).to(torch.int32)[None]
        cache, (q, k, v), angle = run(n, hq, hkv, d, d, 1, False, fp8, positions, slots, pages, g)
        check_stored(cache, k, v, slots, angle, False, fp8)
        # slots that were not given stay as they were: zero
        rest = torch.tensor(sorted(set(range(pages * 16)) - set(slots.tolist())), device="cuda")
        if fp8:
            kc, vc = (torch.ones(rest.numel(), hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2))
            ks, vs = (torch.ones(rest.numel(), hkv, device="cuda") for _ in range(2))
            cache.skv_gather_fp8(0, rest, kc, vc, ks, vs)
            assert not bool(kc.any() or vc.any() or ks.any() or vs.any())
        else:
            ko, vo = (torch.ones(rest.numel(), hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            cache.skv_gather(0, rest, ko, vo)
            assert not bool(ko.any() or vo.any())


def test_far_and_negative_positions():
    """An angle is as good at position 2^31 - 1 as at 1."""
    g = torch.Generator().manual_seed(6)
    far = torch.tensor([0, 1, -1, 1000000, 16777217, 2147483647, -2147483648, 123456789], dtype=torch.int32)[None]
    slots = torch.arange(8)
    for adjacent in (False, True):
        cache, (q, k, v), angle = run(8, 4, 2, 128, 128, 1, adjacent, False, far, slots, 1, g)
        check_stored(cache, k, v, slots, angle, adjacent, False)


def test_special_values_pass():
    """Dims that are not turned and V keep their bits, whatever they are; zeros keep FP8 scale 0."""
    import paper_2604_22782_b200 as skv
    rope = skv.SkvRope(freqs(64), n_axes=1)
    cache = skv.SkvCache([0], 1, 128, 16, 1, allocate=True)
    x = torch.zeros(3, 1, 128, dtype=torch.bfloat16)
    x[0, 0, 64:] = float("inf")
    x[1, 0, 64:] = float("nan")
    x[2, 0, 64:] = -0.0
    xd, out = x.cuda(), torch.empty(3, 1, 128, dtype=torch.bfloat16, device="cuda")
    cache.skv_rope_append(0, rope, xd, out, xd, xd, torch.arange(3, dtype=torch.int32, device="cuda"), torch.arange(3, device="cuda"))
    ko, vo = torch.empty_like(xd), torch.empty_like(xd)
    cache.skv_gather(0, torch.arange(3, device="cuda"), ko, vo)
    for y in (out, ko, vo):
        assert torch.equal(y[..., 64:].cpu().view(torch.int16), x[..., 64:].view(torch.int16))
        assert bool((y[..., :64] == 0).all())
    fp8 = skv.SkvCache([0], 1, 128, 16, 1, allocate=True, fp8=True)
    z = torch.zeros(1, 1, 128, dtype=torch.bfloat16, device="cuda")
    fp8.pool[256:].fill_(0x55)
    fp8.skv_rope_append(0, rope, z, out[:1], z, z, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda"))
    kc, vc = (torch.ones(1, 1, 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.ones(1, 1, device="cuda") for _ in range(2))
    fp8.skv_gather_fp8(0, torch.zeros(1, dtype=torch.int64, device="cuda"), kc, vc, ks, vs)
    assert not bool((kc & 0x7F).any() or (vc & 0x7F).any() or ks.any() or vs.any())


def test_in_place_on_a_fused_projection():
    import paper_2604_22782_b200 as skv
    g = torch.Generator().manual_seed(7)
    n, hq, hkv, d = 77, 8, 2, 128
    rows = torch.randn(n, (hq + 2 * hkv) * d, generator=g).bfloat16()
    dev = rows.cuda()
    cut = lambda x: (x[:, :hq * d].view(n, hq, d), x[:, hq * d:(hq + hkv) * d].view(n, hkv, d), x[:, (hq + hkv) * d:].view(n, hkv, d))  # noqa: E731
    (q, k, v), (qd, kd, vd) = cut(rows), cut(dev)
    cache = skv.SkvCache([0], hkv, d, 16, 10, allocate=True)
    rope = skv.SkvRope(freqs(d))
    slots, pos = torch.arange(n), torch.arange(n, dtype=torch.int32)
    cache.skv_rope_append(0, rope, qd, qd, kd, vd, pos.cuda(), slots.cuda())
    torch.cuda.synchronize()
    angle = ref.angles(pos[None], freqs(d), [0] * (d // 2))
    check_rows(qd, q, angle, False, "queries")
    assert torch.equal(kd.cpu(), k) and torch.equal(vd.cpu(), v)
    check_stored(cache, k, v, slots, angle, False, False)


def test_layers_that_keep_nothing_and_calls_without_queries():
    import paper_2604_22782_b200 as skv
    g = torch.Generator().manual_seed(8)
    n, hq, hkv, d = 20, 8, 2, 128
    slots, pos = torch.arange(n), torch.arange(n, dtype=torch.int32)[None]
    cache, (q, k, v), angle = run(n, hq, hkv, d, d, 1, False, False, pos, slots, 2, g, r=(0, 0), layer=1)
    assert not bool(cache.pool[256:].any())                                      # layer 1 reads layer 0: nothing stored
    rope = skv.SkvRope(freqs(d))
    out = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda")
    cache.skv_rope_append(1, rope, q.cuda(), out, None, None, pos[0].cuda(), None)
    check_rows(out, q, angle, False, "queries of a reading layer")
    before = cache.skv_launch_count()
    cache.skv_rope_append(1, rope, None, None, None, None, pos[0].cuda(), None)   # nothing to do
    empty = torch.empty(0, hq, d, dtype=torch.bfloat16, device="cuda")
    none = torch.empty(0, hkv, d, dtype=torch.bfloat16, device="cuda")
    cache.skv_rope_append(0, rope, empty, empty, none, none, pos[0, :0].cuda(), slots[:0].cuda())
    assert cache.skv_launch_count() == before
    cache.skv_rope_append(0, rope, None, None, k.cuda(), v.cuda(), pos[0].cuda(), slots.cuda())
    check_stored(cache, k, v, slots, angle, False, False)
    cache.skv_rope_append(0, rope, None, None, k.cuda(), v.cuda(), pos[0].cuda(), (slots + 20).cuda())
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    assert cache.skv_get_status() == SKV_ERR_BOUNDS                               # slots 32..39 are beyond two pages
    check_stored(cache, k[:12], v[:12], slots[:12] + 20, angle[:12], False, False)


def test_same_cache_as_rope_and_append_one_after_the_other():
    """On bf16 pages the stored rows are those skv_append would store of the turned rows, bit for bit."""
    import paper_2604_22782_b200 as skv
    g = torch.Generator().manual_seed(9)
    n, hkv, d = 333, 4, 128
    rope = skv.SkvRope(freqs(d))
    k, v = torch.randn(n, hkv, d, generator=g).bfloat16().cuda(), torch.randn(n, hkv, d, generator=g).bfloat16().cuda()
    pos, slots = torch.arange(n, dtype=torch.int32, device="cuda"), torch.randperm(400, generator=g)[:n].cuda()
    one, two = (skv.SkvCache([0], hkv, d, 16, 25, allocate=True) for _ in range(2))
    turned = torch.empty_like(k)
    one.skv_rope_append(0, rope, k, turned, k, v, pos, slots)
    two.skv_append(0, turned, v, slots)
    torch.cuda.synchronize()
    assert torch.equal(one.pool[256:], two.pool[256:])


def test_refusals():
    import paper_2604_22782_b200 as skv
    from paper_2604_22782_b200.binding import SKV_ERR_ARG, SKV_ERR_LAYER, SKV_ERR_UNSUPPORTED, lib
    cache = skv.SkvCache([0, 0], 2, 64, 16, 4, allocate=True)
    rope, wide = skv.SkvRope(freqs(64)), skv.SkvRope(freqs(128))
    q, kv = torch.zeros(4, 4, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos, slots = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.arange(4, device="cuda")
    args = dict(layer=0, rope=rope, q=q.data_ptr(), qs=256, qo=q.data_ptr(), qos=256, k=kv.data_ptr(), ks=128, v=kv.data_ptr(), vs=128,
                pos=pos.data_ptr(), ps=4, slots=slots.data_ptr(), n=4, hq=4)

    def rc(**kw):
        a = dict(args, **kw)
        return lib.skv_rope_append(cache._h, a["layer"], a["rope"]._h if a["rope"] else None, a["q"], a["qs"], a["qo"], a["qos"], a["k"], a["ks"],
                                   a["v"], a["vs"], a["pos"], a["ps"], a["slots"], a["n"], a["hq"], None)

    assert rc(layer=2) == SKV_ERR_LAYER and rc(layer=-1) == SKV_ERR_LAYER
    assert rc(rope=wide) == SKV_ERR_UNSUPPORTED
    for bad in (dict(rope=None), dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(pos=None), dict(slots=None), dict(n=-1), dict(hq=-1),
                dict(qs=255), dict(qs=200), dict(qos=264), dict(ks=64), dict(vs=132), dict(ps=3), dict(q=q.data_ptr() + 2), dict(k=kv.data_ptr() + 8)):
        assert rc(**bad) == SKV_ERR_ARG, bad
    with pytest.raises(ValueError):
        cache.skv_rope_append(0, rope, q, q, kv, kv, pos[None].repeat(3, 1), slots)
    with pytest.raises(ValueError):
        cache.skv_rope_append(0, rope, q.transpose(0, 1), q, kv, kv, pos, slots)
    with pytest.raises(TypeError):
        cache.skv_rope_append(0, rope, q.half(), q, kv, kv, pos, slots)
    with pytest.raises(TypeError):
        cache.skv_rope_append(0, rope, q, q, kv, kv, pos.long(), slots)
    assert cache.skv_launch_count() == 0 and cache.skv_get_status() == 0
