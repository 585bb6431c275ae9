"""A step's tables made on the GPU, number by number against a plain loop over the requests; pages given back; and whole serving
steps (tables, rotary update, windowed attention) over a pool that only suffices because pages come back."""
import pytest
import torch

import serving_reference as ref

pytestmark = pytest.mark.gpu

I32 = torch.int32


def dev(x, dtype=I32):
    return torch.tensor(x, dtype=dtype, device="cuda")


def make(lens, width, spare, g):
    import paper_2604_22782_b200 as skv
    table, total = ref.paged([min(max(n, 0), width * 16) for n in lens], g, spare=spare, width=width)
    used = set(table.flatten().tolist())
    free = [i for i in torch.randperm(total, generator=g).tolist() if i not in used]
    return skv.SkvCache([0], 1, 64, 16, total, allocate=True), table, free


def step(cache, table, lens, new, free, n_free, max_tokens, in_place=False, with_positions=True):
    t, n = table.cuda(), dev(lens)
    slots = torch.full((max_tokens,), -7, dtype=torch.int64, device="cuda")
    pos = torch.full((max_tokens,), -7, dtype=I32, device="cuda")
    cu = torch.full((len(lens) + 1,), -7, dtype=I32, device="cuda")
    left = dev([n_free])
    n_out, left_out = (n, left) if in_place else (torch.empty_like(n), torch.empty_like(left))
    stack = dev(free if free else [0])
    cache.skv_plan_step(t, n, dev(new), stack, left, slots, cu, n_out, left_out, positions=pos if with_positions else None)
    torch.cuda.synchronize()
    assert torch.equal(stack, dev(free if free else [0]))
    return t.cpu(), slots.cpu(), pos.cpu(), cu.cpu(), n_out.cpu(), int(left_out)


def check(cache, table, lens, new, free, n_free, max_tokens, **kw):
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS, SKV_ERR_NOMEM
    want = ref.plan_step(table.tolist(), lens, new, free, n_free, max_tokens)
    t, slots, pos, cu, n_out, left = step(cache, table, lens, new, free, n_free, max_tokens, **kw)
    m = want[3][-1]
    assert t.tolist() == want[0] and cu.tolist() == want[3] and n_out.tolist() == want[4] and left == want[5]
    assert slots[:m].tolist() == want[1] and bool((slots[m:] == -7).all())
    if kw.get("with_positions", True):
        assert pos[:m].tolist() == want[2] and bool((pos[m:] == -7).all())
    row = table.shape[1] * 16
    status = cache.skv_get_status()
    if any(max(lens[b], 0) + new[b] > row for b in want[6]):
        assert status == SKV_ERR_BOUNDS
    else:
        assert status == (SKV_ERR_NOMEM if want[6] else 0)
    return t, n_out.tolist(), left


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch", [1, 2, 31, 33, 256, 257, 1025, 5000])
def test_ragged_requests(batch, in_place):
    g = torch.Generator().manual_seed(batch)
    width = 20
    lens = torch.randint(0, 200, (batch,), generator=g).tolist()
    for most in (1, 5, 100):
        new = torch.randint(0, most + 1, (batch,), generator=g).tolist()
        need = sum(-(-(n + a) // 16) - -(-n // 16) for n, a in zip(lens, new))
        cache, table, free = make(lens, width, need + 5, g)
        total = max(1, sum(new))
        check(cache, table, lens, new, free, len(free), total + 3, in_place=in_place)
        check(cache, table, lens, new, free, need, total, in_place=in_place)                     # just enough
        if need:
            check(cache, table, lens, new, free, need - 1, total, in_place=in_place)             # the last ones have to wait
            check(cache, table, lens, new, free, need // 3, total, in_place=in_place)
        check(cache, table, lens, new, free, len(free), max(1, total // 2), in_place=in_place)   # no room for all tokens
        check(cache, table, lens, new, free, 0, total, in_place=in_place, with_positions=False)


def test_edges():
    g = torch.Generator().manual_seed(1)
    lens, new = [0, 16, 15, 0, 320, 319, 320, 5], [0, 16, 1, 1, 0, 1, 1, -3]
    cache, table, free = make(lens, 20, 40, g)
    check(cache, table, lens, new, free, len(free), 100)          # the seventh does not fit its row of 20 pages
    check(cache, table, lens, new, free, -5, 100)                 # a count below zero: no pages
    check(cache, table, lens, new, free, len(free) + 9, 100)      # a count beyond the stack: the stack
    check(cache, table, lens, [0] * 8, free, len(free), 1)        # nothing wanted
    check(cache, table, [n if n >= 0 else 0 for n in lens], [1 << 30] * 8, free, len(free), 100)


def test_negative_lengths_count_as_zero():
    g = torch.Generator().manual_seed(2)
    cache, table, free = make([0, 0, 3], 4, 9, g)
    check(cache, table, [-4, 0, 3], [3, 2, -9], free, len(free), 100)


def test_many_tokens_over_many_blocks():
    g = torch.Generator().manual_seed(3)
    lens = [5, 0, 17, 100000, 0, 3]
    new = [40000, 0, 33333, 7, 120000, 1]
    cache, table, free = make(lens, 8000, 13000, g)
    for in_place in (False, True):
        check(cache, table, lens, new, free, len(free), 200000, in_place=in_place)


def test_bad_page_ids_are_flagged_not_written():
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    g = torch.Generator().manual_seed(4)
    cache, table, free = make([5, 20], 4, 4, g)
    table[0, 0] = 1 << 30
    t, slots, pos, cu, n_out, left = step(cache, table, [5, 20], [3, 2], free, len(free), 5)
    assert cache.skv_get_status() == SKV_ERR_BOUNDS
    assert slots[:3].tolist() == [-1] * 3 and bool((slots[3:] >= 0).all())


def test_largest_batch_and_refusals():
    import paper_2604_22782_b200 as skv
    from paper_2604_22782_b200.binding import SKV_ERR_ARG, SKV_ERR_UNSUPPORTED, lib
    g = torch.Generator().manual_seed(5)
    batch = 16384
    lens = torch.randint(0, 60, (batch,), generator=g).tolist()
    cache, table, free = make(lens, 5, batch, g)
    for in_place in (False, True):
        check(cache, table, lens, [1] * batch, free, len(free), batch, in_place=in_place)
    small = skv.SkvCache([0], 1, 64, 16, 4, allocate=True)
    b = torch.zeros(64, dtype=I32, device="cuda").data_ptr()
    ok = dict(table=b, width=4, n=b, new=b, batch=2, free=b, cap=4, nf=b, m=4, slots=b, pos=b, cu=b, out=b, nfo=b)

    def rc(**kw):
        a = dict(ok, **kw)
        return lib.skv_plan_step(small._h, a["table"], a["width"], a["n"], a["new"], a["batch"], a["free"], a["cap"], a["nf"], a["m"], a["slots"],
                                 a["pos"], a["cu"], a["out"], a["nfo"], None)

    assert rc(batch=16385) == SKV_ERR_UNSUPPORTED
    for bad in (dict(batch=0), dict(width=0), dict(cap=-1), dict(m=-1), dict(m=1 << 31), dict(table=None), dict(n=None), dict(new=None),
                dict(free=None), dict(nf=None), dict(slots=None), dict(cu=None), dict(out=None), dict(nfo=None)):
        assert rc(**bad) == SKV_ERR_ARG, bad
    rel = lambda **kw: (lambda a: lib.skv_plan_release(small._h, a["table"], a["width"], a["n"], a["new"], a["batch"], a["free"], a["cap"], a["nf"], a["nfo"], None))(dict(ok, **kw))  # noqa: E731
    assert rel(batch=16385) == SKV_ERR_UNSUPPORTED
    for bad in (dict(batch=0), dict(width=0), dict(cap=-1), dict(table=None), dict(n=None), dict(new=None), dict(free=None), dict(nf=None), dict(nfo=None)):
        assert rel(**bad) == SKV_ERR_ARG, bad
    with pytest.raises(ValueError):
        small.skv_plan_step(dev([[0]]), dev([1, 2]), dev([1, 1]), dev([0]), dev([0]), dev([0], torch.int64), dev([0] * 3), dev([0, 0]), dev([0]))
    with pytest.raises(TypeError):
        small.skv_plan_release(dev([[0]]), dev([0], torch.int64), dev([1]), dev([0]), dev([0]), dev([0]))
    assert small.skv_launch_count() == 0


@pytest.mark.parametrize("batch", [1, 40, 1500, 16384])
def test_release(batch):
    from paper_2604_22782_b200.binding import SKV_ERR_NOMEM
    g = torch.Generator().manual_seed(batch)
    lens = torch.randint(0, 700, (batch,), generator=g).tolist()
    cache, table, free = make(lens, 45, 6, g)
    first = torch.randint(-3, 40, (batch,), generator=g).tolist()
    end = torch.randint(-3, 60, (batch,), generator=g).tolist()
    table[:, 3] = -1                                              # given back before
    for room in (1 << 30, 5):
        want_t, want_s, held = [list(r) for r in table.tolist()], list(free), 0
        for b in range(batch):
            for p in range(max(first[b], 0), min(end[b], 45)):
                if want_t[b][p] >= 0:
                    held += 1
                    if len(want_s) < min(len(free) + room, len(free) + held):
                        want_s.append(want_t[b][p])
                        want_t[b][p] = -1
        cap = len(free) + min(room, batch * 45)
        t, stack = table.cuda(), torch.full((cap,), -7, dtype=I32, device="cuda")
        stack[:len(free)] = dev(free)
        left = dev([len(free)])
        cache.skv_plan_release(t, dev(first), dev(end), stack, left, left)
        torch.cuda.synchronize()
        assert int(left) == len(want_s) and stack[:len(want_s)].tolist() == want_s and t.tolist() == want_t
        assert cache.skv_get_status() == (SKV_ERR_NOMEM if held > room else 0)


def test_release_flags_ids_beyond_the_pool():
    from paper_2604_22782_b200.binding import SKV_ERR_BOUNDS
    g = torch.Generator().manual_seed(6)
    cache, table, free = make([40], 4, 2, g)
    table[0, 1] = 1 << 29
    t, stack, left = table.cuda(), torch.zeros(10, dtype=I32, device="cuda"), dev([0])
    cache.skv_plan_release(t, dev([0]), dev([4]), stack, left, left)
    assert cache.skv_get_status() == SKV_ERR_BOUNDS and int(left) == 2
    assert t.tolist() == [[-1, 1 << 29, -1, -1]] and stack[:2].tolist() == [int(table[0, 0]), int(table[0, 2])]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_serving_steps_in_a_pool_that_pages_come_back_to(hq, hkv, d, fp8):
    """Prompts in chunks, then tokens one by one, in place and without the host looking at a number: tables, rotary
    update and windowed attention of every layer, then the pages that the windows have left go back.  The pool holds a
    quarter of what the sequences come to."""
    import paper_2604_22782_b200 as skv
    window, sinks, r = 70, 5, [0, 0, 2]
    batch, width, pages = 3, 64, 48
    cache = skv.SkvCache(r, hkv, d, 16, pages, allocate=True, fp8=fp8)
    inv = [1e4 ** (-2.0 * i / d) for i in range(d // 2)]
    rope = skv.SkvRope(inv)
    g = torch.Generator().manual_seed(7)
    table = torch.full((batch, width), -1, dtype=I32, device="cuda")
    lens, left = torch.zeros(batch, dtype=I32, device="cuda"), dev([pages])
    stack = torch.randperm(pages, generator=g).to(I32).cuda()
    ws = torch.empty(cache.skv_decode_workspace_bytes(batch, hq), dtype=torch.uint8, device="cuda")
    plan = [[90, 33, 1], [64, 64, 64], [0, 100, 17], [100, 0, 64], [100, 64, 64]] + [[1, 1, 1]] * 20 + [[90, 64, 64]] * 4 + [[1, 0, 1]] * 3
    hist = {l: ([torch.zeros(0, hkv, d)] * batch, [torch.zeros(0, hkv, d)] * batch) for l in (0, 2)}
    n_host = [0] * batch
    for new in plan:
        m = sum(new)
        slots = torch.full((m + 2,), -1, dtype=torch.int64, device="cuda")
        pos = torch.zeros(m + 2, dtype=I32, device="cuda")
        cu = torch.zeros(batch + 1, dtype=I32, device="cuda")
        cache.skv_plan_step(table, lens, dev(new), stack, left, slots, cu, lens, left, positions=pos)
        n_host = [n + a for n, a in zip(n_host, new)]
        for layer in range(3):
            q, k, v = (torch.randn(m, h, d, generator=g).bfloat16() for h in (hq, hkv, hkv))
            qd, out = torch.empty(m, hq, d, dtype=torch.bfloat16, device="cuda"), torch.full((m, hq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
            cache.skv_rope_append(layer, rope, q.cuda(), qd, k.cuda(), v.cuda(), pos[:m], slots[:m])
            if new == [1, 1, 1]:
                cache.skv_decode_attn_window(layer, qd, table, lens, out, ws, window, sinks)
            else:
                cache.skv_prefill_attn_window(layer, qd, cu, table, lens, out, max(new), window, sinks)
            if r[layer] == layer:
                # what the pages hold of the new tokens, read back: the attention is held to that
                ids = slots[:m]
                if fp8:
                    kc, vc = (torch.empty(m, hkv, d, dtype=torch.uint8, device="cuda") for _ in range(2))
                    ks, vs = (torch.empty(m, hkv, device="cuda") for _ in range(2))
                    cache.skv_gather_fp8(layer, ids, kc, vc, ks, vs)
                    rows = [(c.view(torch.float8_e4m3fn).double() * s.double()[..., None]).cpu() for c, s in ((kc, ks), (vc, vs))]
                else:
                    rows = [torch.empty(m, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
                    cache.skv_gather(layer, ids, *rows)
                    rows = [x.double().cpu() for x in rows]
                for i in range(2):
                    parts = torch.split(rows[i], new)
                    hist[layer] = tuple([torch.cat((a, b)) for a, b in zip(hist[layer][j], parts)] if j == i else hist[layer][j] for j in range(2))
            angle = ref.angles(torch.cat([torch.arange(n - a, n) for n, a in zip(n_host, new)])[None], inv, [0] * (d // 2))
            turned, size = ref.rope(q, angle, False)
            assert bool(((qd.double().cpu() - turned).abs() <= ref.rope_tolerance(turned, size)).all())
            row = 0
            for b, (n, a) in enumerate(zip(n_host, new)):
                ks, vs = hist[r[layer]][0][b], hist[r[layer]][1][b]
                o, size, reach = ref.attention(qd[row:row + a].cpu(), ks, vs, torch.arange(n - a, n), window, sinks)
                tol = ref.attention_tolerance(o, size, reach, n, fp8, float(vs.abs().max()) if n else 0.0)
                assert bool(((out[row:row + a].double().cpu() - o).abs() <= tol).all()), (layer, b, n)
                row += a
        # the next row is at position n: it sees n - window + 1 .. n and the sinks
        gone = ((lens - window + 1).clamp(min=0) // 16).to(I32)
        cache.skv_plan_release(table, torch.full_like(gone, -(-sinks // 16)), gone, stack, left, left)
        assert lens.tolist() == n_host
        held = [int((table[b] >= 0).sum()) for b in range(batch)]
        assert int(left) == pages - sum(held) and all(h <= 1 + -(-(window + 15) // 16) + 1 for h in held)
        everything = sorted(stack[:int(left)].tolist() + [x for x in table.flatten().tolist() if x >= 0])
        assert everything == list(range(pages))                   # no page lost, none given out twice
    assert sum(n_host) > pages * 16 and cache.skv_get_status() == 0


def test_a_captured_step_advances_at_every_replay():
    """Lengths and stack in place: the graph of one step, replayed, walks through positions and pages."""
    import paper_2604_22782_b200 as skv
    cache = skv.SkvCache([0], 1, 64, 16, 12, allocate=True)
    table, lens, left = torch.full((2, 6), -1, dtype=I32, device="cuda"), dev([0, 14]), dev([11])
    table[1, 0] = 11
    stack, new = dev(list(range(11))), dev([1, 2])
    slots, pos, cu = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=I32, device="cuda"), torch.zeros(3, dtype=I32, device="cuda")
    host = [[-1] * 6, [11] + [-1] * 5], [0, 14], 11
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            cache.skv_plan_step(table, lens, new, stack, left, slots, cu, lens, left, positions=pos)
    for _ in range(30):
        g.replay()
        torch.cuda.synchronize()
        t, sl, po, c, n, nf, refused = ref.plan_step(host[0], host[1], [1, 2], list(range(11)), host[2], 3)
        assert table.tolist() == t and lens.tolist() == n and int(left) == nf and slots[:c[-1]].tolist() == sl and pos[:c[-1]].tolist() == po
        host = t, n, nf
    assert cache.skv_get_status() == 0
