"""What is measured of the serving-step operators: attention over a sliding window with sinks (decode and chunk), rotary
embedding with the update of the cache, and the page tables and slot maps of a step.

Each operator has a plain form in elementary torch operations and the call a user makes of the library.  Both work on the
same state: the page pool is laid out as the library lays it out (a plain tensor here), so neither side converts anything
that the other does not."""
import math

import torch

own = False

PAGE = 16
HEADER = 256            # bytes before the first page of a pool


# ---- cases -------------------------------------------------------------------------------------------------------
def _decode(name, batch, hq, hkv, d, lo, hi, window, sinks, fp8=False, full=False):
    return {"name": name, "op": "decode", "batch": batch, "hq": hq, "hkv": hkv, "d": d, "lo": lo, "hi": hi, "window": window,
            "sinks": sinks, "fp8": fp8, "full": full}


def _chunk(name, batch, hq, hkv, d, q_lo, q_hi, before, window, sinks, fp8=False):
    return {"name": name, "op": "chunk", "batch": batch, "hq": hq, "hkv": hkv, "d": d, "q_lo": q_lo, "q_hi": q_hi, "before": before,
            "window": window, "sinks": sinks, "fp8": fp8}


def _rope(name, tokens, hq, hkv, d, rotary, axes, theta, far, fp8=False, adjacent=False):
    return {"name": name, "op": "rope", "tokens": tokens, "hq": hq, "hkv": hkv, "d": d, "rotary": rotary, "axes": axes, "theta": theta,
            "far": far, "fp8": fp8, "adjacent": adjacent}


def _plan(name, batch, lo, hi, new_lo, new_hi, width, short=False):
    return {"name": name, "op": "plan", "batch": batch, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "width": width, "short": short}


def listed():
    return [
        # one user's token on a grouped-query model with a 1 K window: nothing but latency
        _decode("decode_1_w1024", 1, 32, 8, 128, 8320, 8320, 1024, 4),
        # a mid-sized batch, some sequences shorter than the window; all pages still held by the table
        _decode("decode_32_w2048", 32, 32, 8, 128, 1024, 8192, 2048, 4, full=True),
        # one query head per kv head at long context; the pool passes 4 GiB
        _decode("decode_mha_32k_w4096", 8, 32, 32, 128, 32768, 32768, 4096, 16, full=True),
        # a full server on FP8 pages
        _decode("decode_128_fp8_w4096", 128, 32, 8, 128, 2048, 16384, 4096, 4, fp8=True),
        # two prompts in whole, window half their length
        _chunk("chunk_2x4096_w2048", 2, 32, 8, 128, 4096, 4096, 0, 2048, 4),
        # a step of chunked prompts behind long histories, ragged
        _chunk("chunk_8x512_w1024", 8, 32, 8, 128, 257, 512, 6000, 1024, 4),
        # short ragged chunks at head_dim 64 with three query heads per kv head, odd window, no sinks
        _chunk("chunk_5_d64_w300", 5, 6, 2, 64, 1, 130, 1000, 300, 0),
        # the decode step's tokens
        _rope("rope_64", 64, 32, 8, 128, 128, 1, 5e5, 32768),
        # image and text tokens of a prompt with three position axes
        _rope("rope_8191_axes3", 8191, 32, 8, 128, 128, 3, 1e6, 32768),
        # long prompts onto FP8 pages
        _rope("rope_32768_fp8", 32768, 32, 8, 128, 128, 1, 5e5, 1 << 20, fp8=True),
        # a decode step of a server
        _plan("plan_64_step", 64, 1024, 4096, 1, 1, 520),
        # prompts and steps mixed
        _plan("plan_256_mixed", 256, 0, 4096, 1, 255, 520),
    ]


HEADS = [(32, 8, 128), (32, 32, 128), (8, 1, 128), (4, 4, 128), (6, 2, 128), (8, 2, 128), (4, 2, 64), (6, 2, 64)]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["decode", "decode", "chunk", "chunk", "rope", "plan"])
    if op == "decode":
        hq, hkv, d = rng.choice(HEADS)
        hi = _log(rng, 1, 32768)
        lo = rng.randint(0, hi)
        window, sinks = _log(rng, 1, 8192), rng.choice([0, 1, 4, rng.randint(2, 70)])
        most = 120_000_000 // (hkv * d * min(hi, window + sinks + 16))
        batch = _log(rng, 1, max(1, min(128, most, 400_000_000 // (hkv * d * hi))))
        c = _decode("", batch, hq, hkv, d, lo, hi, window, sinks, fp8=rng.random() < 0.4, full=rng.random() < 0.5)
    elif op == "chunk":
        hq, hkv, d = rng.choice(HEADS)
        q_hi = _log(rng, 1, 3000)
        window, sinks = _log(rng, 1, 4096), rng.choice([0, 4, rng.randint(1, 70)])
        before = rng.choice([0, _log(rng, 1, 8192)])
        most = 1_000_000_000 // (hq * q_hi * (q_hi + min(before, window) + sinks))
        c = _chunk("", _log(rng, 1, max(1, min(16, most))), hq, hkv, d, rng.randint(1, q_hi), q_hi, before, window, sinks, fp8=rng.random() < 0.3)
    elif op == "rope":
        hq, hkv, d = rng.choice(HEADS)
        n = _log(rng, 1, 20000)
        c = _rope("", n, hq, hkv, d, rng.choice([d, d, d // 2]), rng.choice([1, 3]), rng.choice([1e4, 5e5, 1e6]), _log(rng, 100, 1 << 22),
                  fp8=rng.random() < 0.3, adjacent=rng.random() < 0.3)
    else:
        batch = _log(rng, 1, 500)
        new_hi = _log(rng, 1, max(1, 60000 // batch))
        hi = rng.randint(0, 8000)
        c = _plan("", batch, rng.randint(0, hi), hi, rng.randint(0, new_hi), new_hi, (hi + new_hi) // PAGE + rng.randint(1, 9), short=rng.random() < 0.3)
    del c["name"]
    return c


# ---- sizes that follow from a case ---------------------------------------------------------------------------------
def _spread(lo, hi, n, salt):
    """n whole numbers of [lo, hi], the first of them hi, the same ones for a case every time."""
    return [hi if i == 0 else lo + ((i + salt) * 2654435761 % 4294967296) * (hi - lo + 1) // 4294967296 for i in range(n)]


def _lens(c):
    """(cached tokens, new tokens) of every sequence, the new ones counted among the cached ones for the attentions."""
    if c["op"] == "decode":
        n = _spread(c["lo"], c["hi"], c["batch"], 1)
        return n, [1] * c["batch"]
    if c["op"] == "chunk":
        q = _spread(c["q_lo"], c["q_hi"], c["batch"], 1)
        return [x + y for x, y in zip(_spread(c["before"] // 2, c["before"], c["batch"], 7), q)], q
    return _spread(c["lo"], c["hi"], c["batch"], 1), _spread(c["new_lo"], c["new_hi"], c["batch"], 5)


def _seen(c):
    """Per sequence: (tokens that some row sees, visible pairs of row and token)."""
    w, s, got = c["window"], c["sinks"], []
    for n, q in zip(*_lens(c)):
        if n == 0:
            got.append((0, 0))
            continue
        lo = max(0, n - q - w + 1)                       # first token inside some row's window
        tokens = n - lo + min(s, lo)
        pos = torch.arange(n - q, n, dtype=torch.int64)
        first = (pos - w + 1).clamp(min=0)
        got.append((tokens, int((pos + 1 - first + first.clamp(max=s)).sum())))
    return got


def work(case):
    c = case
    if c["op"] in ("decode", "chunk"):
        seen, rows = _seen(c), sum(_lens(c)[1])
        row = c["d"] + 4 if c["fp8"] else 2 * c["d"]
        return {"bytes": sum(t for t, _ in seen) * c["hkv"] * 2 * row + 4 * rows * c["hq"] * c["d"] + 4 * 2 * c["batch"],
                "flops": 4 * c["d"] * c["hq"] * sum(p for _, p in seen)}
    if c["op"] == "rope":
        kept = 2 * (c["d"] + 4) if c["fp8"] else 4 * c["d"]
        n = c["tokens"]
        return {"bytes": n * (4 * c["hq"] * c["d"] + c["hkv"] * (4 * c["d"] + kept) + 4 * c["axes"] + 8),
                "flops": n * 3 * c["rotary"] * (c["hq"] + c["hkv"])}
    new, pages = sum(_lens(c)[1]), 0
    for n, a in zip(*_lens(c)):
        pages += (n + a + PAGE - 1) // PAGE - (n + PAGE - 1) // PAGE
    # slot and position of every token, a page id read and written for every new page, the requests' lengths in and out
    return {"bytes": 12 * new + 8 * pages + 16 * c["batch"], "flops": 0}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _table(c, g, dev):
    """(page table, pages of the pool): pages in a random order; where the pool is not held in full, those that no row of the
    call sees have been given back and their entries are -1."""
    n, q = _lens(c)
    width = max(1, (max(n) + PAGE - 1) // PAGE)
    n, q = (torch.tensor(x, device=dev) for x in (n, q))
    p = torch.arange(width, device=dev)[None]
    held = p * PAGE < n[:, None]
    if not c.get("full"):
        lo = (n - q - c["window"] + 1).clamp(min=0)
        held &= ((p + 1) * PAGE > lo[:, None]) | (p * PAGE < c["sinks"])
    total = max(1, int(held.sum()))
    table = torch.full((len(n), width), -1, dtype=torch.int32, device=dev)
    table[held] = torch.randperm(total, generator=g, device=dev)[: int(held.sum())].to(torch.int32)
    return table, total


def _pool(c, pages, dev):
    """Zeroed bytes of a pool of one owner layer and what it holds, as views: bf16 [page][head][K|V][chunk of 8][token][8]; on FP8 pages
    the codes of K [page][head][8-token group][chunk of 16][token][16] and of V [page][head][dim][token] and the scales [page][head][K|V][token]."""
    h, d = c["hkv"], c["d"]
    block = 2 * PAGE * (d + 4) if c["fp8"] else 4 * PAGE * d
    pool = torch.zeros(HEADER + pages * h * block, dtype=torch.uint8, device=dev)
    body = pool[HEADER:].view(pages, h, block)
    if not c["fp8"]:
        return pool, (body.view(torch.bfloat16).view(pages, h, 2, d // 8, PAGE, 8),)
    half = PAGE * d
    return pool, (body[..., :half].unflatten(2, (2, d // 16, 8, 16)).view(torch.float8_e4m3fn), body[..., half:2 * half].unflatten(2, (d, PAGE)).view(torch.float8_e4m3fn),
                  body.view(torch.float32)[..., half // 2:].unflatten(2, (2, PAGE)))


def _quantised(x):
    """E4M3 codes and the scale of every row of the last dimension."""
    amax = x.abs().amax(-1, keepdim=True)
    codes = (x * torch.where(amax > 0, 448.0 / amax, torch.zeros_like(amax))).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)
    return codes, (amax / 448.0)[..., 0]


def _fill(c, held, g, dev):
    """Keys and values of every slot: what projections of normalised activations look like."""
    if not c["fp8"]:
        held[0].normal_(generator=g)
        return
    pages, h, d = held[1].shape[0], c["hkv"], c["d"]
    k, ks = _quantised(torch.randn((pages, h, PAGE, d), generator=g, device=dev))
    v, vs = _quantised(torch.randn((pages, h, PAGE, d), generator=g, device=dev))
    u = torch.uint8
    held[0].view(u).copy_(k.view(u).view(pages, h, 2, 8, d // 16, 16).transpose(3, 4))
    held[1].view(u).copy_(v.view(u).transpose(2, 3))
    held[2].copy_(torch.stack((ks, vs), 2))


def _axis_of(c):
    """Which position axis turns frequency i: one, or time, height and width in runs of 2 : 3 : 3."""
    half = c["rotary"] // 2
    if c["axes"] == 1:
        return [0] * half
    return [0 if i < half // 4 else 1 if i < half // 4 + half * 3 // 8 else 2 for i in range(half)]


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    s = {"case": c}
    if own:
        import paper_2604_22782_b200 as skv
    if c["op"] == "plan":
        n, a = _lens(c)
        width, need = c["width"], sum((x + y + PAGE - 1) // PAGE - (x + PAGE - 1) // PAGE for x, y in zip(n, a))
        used = sum((x + PAGE - 1) // PAGE for x in n)
        spare = need // 2 if c["short"] else need + 8    # (short: requests at the end of the batch have to wait)
        total = max(1, used + spare)
        s["n"], s["new"] = (torch.tensor(x, dtype=torch.int32, device=dev) for x in (n, a))
        ids = torch.randperm(total, generator=g, device=dev).to(torch.int32)
        held = torch.arange(width, device=dev)[None] * PAGE < s["n"][:, None]
        s["table"] = torch.full((c["batch"], width), -1, dtype=torch.int32, device=dev)
        s["table"][held] = ids[:used]
        s["free"] = ids[used:used + max(1, spare)].contiguous() if spare else torch.zeros(1, dtype=torch.int32, device=dev)
        s["n_free"] = torch.tensor([spare], dtype=torch.int32, device=dev)
        s["tokens"] = max(1, sum(a))
        s["slots"] = torch.full((s["tokens"],), -1, dtype=torch.int64, device=dev)
        s["pos"] = torch.full((s["tokens"],), -1, dtype=torch.int32, device=dev)
        s["cu"] = torch.zeros(c["batch"] + 1, dtype=torch.int32, device=dev)
        s["n_out"], s["n_free_out"] = torch.zeros_like(s["n"]), torch.zeros_like(s["n_free"])
        if own:
            s["cache"] = skv.SkvCache([0], 2, 64, PAGE, total, allocate=True)
        return s
    if c["op"] == "rope":
        t, hq, hkv, d = c["tokens"], c["hq"], c["hkv"], c["d"]
        pages = (t + PAGE - 1) // PAGE
    else:
        s["table"], pages = _table(c, g, dev)
    s["pool"], s["held"] = _pool(c, pages, dev)
    if own:
        s["cache"] = skv.SkvCache([0], c["hkv"], c["d"], PAGE, pages, device_pool=s["pool"], fp8=c["fp8"])
    if c["op"] == "rope":
        qkv = torch.randn((t, (hq + 2 * hkv) * d), generator=g, device=dev).to(torch.bfloat16)      # a fused projection's rows
        s["q"] = qkv[:, :hq * d].view(t, hq, d)
        s["k"] = qkv[:, hq * d:(hq + hkv) * d].view(t, hkv, d)
        s["v"] = qkv[:, (hq + hkv) * d:].view(t, hkv, d)
        first = torch.randint(0, c["far"], (1,), generator=g, device=dev)
        s["pos"] = torch.stack([first + torch.arange(t, device=dev) // 3 ** i for i in range(c["axes"])]).to(torch.int32)
        order = torch.randperm(pages, generator=g, device=dev)
        at = torch.arange(t, device=dev)
        s["slots"] = order[at // PAGE] * PAGE + at % PAGE
        half = c["rotary"] // 2
        s["freq"] = [c["theta"] ** (-i / half) for i in range(half)]
        s["freq_dev"] = torch.tensor(s["freq"], dtype=torch.float64, device=dev)
        s["axis"] = torch.tensor(_axis_of(c), device=dev)
        if own:
            s["rope"] = skv.SkvRope(s["freq"], axis=_axis_of(c), n_axes=c["axes"], adjacent_pairs=c["adjacent"])
        return s
    _fill(c, s["held"], g, dev)
    n, q = _lens(c)
    s["n"] = torch.tensor(n, dtype=torch.int32, device=dev)
    s["q"] = torch.randn((sum(q), c["hq"], c["d"]), generator=g, device=dev).to(torch.bfloat16)
    if c["op"] == "chunk":
        s["cu"] = torch.tensor([0] + torch.tensor(q).cumsum(0).tolist(), dtype=torch.int32, device=dev)
        s["q_most"] = max(q)
        s["reach"] = max(min(x, y + c["window"] - 1) for x, y in zip(n, q))      # tokens inside some row's window, at most
    elif own:
        s["work"] = torch.empty(s["cache"].skv_decode_workspace_bytes(c["batch"], c["hq"]), dtype=torch.uint8, device=dev)
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def _rows(s, t):
    """K and V of tokens t [batch][m] in 32 bits, [batch][m][head][dim]; a token that is not there (t < 0) reads as zero."""
    c, held = s["case"], s["held"]
    b, m = t.shape
    live = (t >= 0)[..., None, None]
    t = t.clamp(min=0)
    page = s["table"].gather(1, t // PAGE).long().clamp(min=0)
    at = t % PAGE
    if c["fp8"]:
        u = torch.uint8
        k = held[0].view(u)[page, :, at // 8, :, at % 8].view(torch.float8_e4m3fn).float().reshape(b, m, c["hkv"], c["d"]) * held[2][page, :, 0, at][..., None]
        v = held[1].view(u)[page, :, :, at].view(torch.float8_e4m3fn).float() * held[2][page, :, 1, at][..., None]
    else:
        k = held[0][page, :, 0, :, at].float().reshape(b, m, c["hkv"], c["d"])
        v = held[0][page, :, 1, :, at].float().reshape(b, m, c["hkv"], c["d"])
    return torch.where(live, k, 0.0), torch.where(live, v, 0.0)


def _softmax_of_seen(x, seen):
    """Softmax over the last dimension among the seen tokens; a row that sees none is zero."""
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total))


def _decode_plain(s):
    c, q, n = s["case"], s["q"], s["n"].long()[:, None]
    most = min(c["window"], c["hi"])
    first = (n - c["window"]).clamp(min=0)
    sink = torch.arange(min(c["sinks"], c["hi"]), device=q.device)[None].expand(len(n), -1)
    t = torch.cat((torch.where(sink < first, sink, -1), first + torch.arange(most, device=q.device)[None]), 1)
    t = torch.where(t < n, t, -1)
    k, v = _rows(s, t)
    qg = q.float().view(len(n), c["hkv"], -1, c["d"])
    x = torch.matmul(qg, k.permute(0, 2, 3, 1)) / math.sqrt(c["d"])
    p = _softmax_of_seen(x, (t >= 0)[:, None, None])
    return torch.matmul(p, v.transpose(1, 2)).reshape(q.shape).to(torch.bfloat16)


def _chunk_plain(s):
    c, q, dev = s["case"], s["q"], s["q"].device
    n, cu = s["n"].long()[:, None], s["cu"].long()
    batch, rows = len(n), s["q_most"]
    new = (cu[1:] - cu[:-1])[:, None]
    i = torch.arange(rows, device=dev)[None]
    row = (cu[:-1, None] + i).clamp(max=len(q) - 1)
    pos = n - new + i                                                        # [batch][rows]
    first = (n - new - c["window"] + 1).clamp(min=0)
    sink = torch.arange(c["sinks"], device=dev)[None].expand(batch, -1)
    t = torch.cat((torch.where(sink < first, sink, -1), first + torch.arange(s["reach"], device=dev)[None]), 1)
    t = torch.where(t < n, t, -1)
    k, v = _rows(s, t)
    qg = q.float()[row].view(batch, rows, c["hkv"], -1, c["d"]).permute(0, 2, 3, 1, 4).flatten(2, 3)       # [batch][head][group x rows][dim]
    x = torch.matmul(qg, k.permute(0, 2, 3, 1)) / math.sqrt(c["d"])
    key, at = t[:, None], pos[..., None]
    seen = (key >= 0) & (key <= at) & ((key > at - c["window"]) | (key < c["sinks"]))                      # [batch][rows][tokens]
    p = _softmax_of_seen(x.unflatten(2, (-1, rows)), seen[:, None, None]).flatten(2, 3)
    o = torch.matmul(p, v.transpose(1, 2)).unflatten(2, (-1, rows)).permute(0, 3, 1, 2, 4).reshape(batch, rows, c["hq"], c["d"])
    return o[i.expand(batch, -1) < new].to(torch.bfloat16)


def _turned(x, cos, sin, rotary, adjacent):
    """Rotary embedding of [token][head][dim] in 32 bits."""
    x, rest = x.float()[..., :rotary], x.float()[..., rotary:]
    a, b = (x[..., 0::2], x[..., 1::2]) if adjacent else x.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if adjacent else torch.cat((a, b), -1), rest), -1)


def _rope_plain(s):
    c, held, d = s["case"], s["held"], s["case"]["d"]
    angle = s["pos"].double()[s["axis"]].t() * s["freq_dev"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _turned(s["q"], cos, sin, c["rotary"], c["adjacent"]).to(torch.bfloat16)
    k = _turned(s["k"], cos, sin, c["rotary"], c["adjacent"])
    t, page, at = len(k), s["slots"] // PAGE, s["slots"] % PAGE
    if c["fp8"]:
        u = torch.uint8
        kc, ks = _quantised(k)
        vc, vs = _quantised(s["v"].float())
        held[0].view(u)[page, :, at // 8, :, at % 8] = kc.view(u).view(t, c["hkv"], d // 16, 16)
        held[1].view(u)[page, :, :, at] = vc.view(u)
        held[2][page, :, 0, at] = ks
        held[2][page, :, 1, at] = vs
    else:
        held[0][page, :, 0, :, at] = k.to(torch.bfloat16).view(t, c["hkv"], d // 8, 8)
        held[0][page, :, 1, :, at] = s["v"].reshape(t, c["hkv"], d // 8, 8)
    return (q,) + held


def _plan_plain(s):
    c, table, dev = s["case"], s["table"], s["table"].device
    n, a, spare = s["n"].long(), s["new"].long(), s["n_free"].long()
    pages = lambda x: (x + PAGE - 1) // PAGE  # noqa: E731
    need = pages(n + a) - pages(n)
    ok = ((need.cumsum(0) <= spare) | (need == 0)) & (a.cumsum(0) <= s["tokens"]) & (n + a <= table.shape[1] * PAGE)
    a, need = torch.where(ok, a, 0), torch.where(ok, need, 0)
    s["cu"][1:] = a.cumsum(0)
    s["n_out"].copy_(n + a)
    s["n_free_out"].copy_(spare - need.sum())
    # the pages of a request come off the top of the stack, in request order
    p, before = torch.arange(table.shape[1], device=dev)[None], (need.cumsum(0) - need)[:, None]
    nth = before + p - pages(n)[:, None]
    fresh = (p >= pages(n)[:, None]) & (p < pages(n + a)[:, None])
    table.copy_(torch.where(fresh, s["free"][(spare - 1 - nth).clamp(0, len(s["free"]) - 1)], table))
    i = torch.arange(s["tokens"], device=dev)
    cu = s["cu"].long()
    b = torch.searchsorted(cu, i, right=True).sub(1).clamp(max=c["batch"] - 1)
    pos = n[b] + i - cu[b]
    there = i < cu[-1]
    slot = table[b, (pos // PAGE).clamp(max=table.shape[1] - 1)].long() * PAGE + pos % PAGE
    s["slots"].copy_(torch.where(there, slot, s["slots"]))
    s["pos"].copy_(torch.where(there, pos, s["pos"].long()))
    return _planned(s)


def _planned(s):
    return s["table"], s["slots"], s["pos"], s["cu"], s["n_out"], s["n_free_out"]


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"decode": _decode_plain, "chunk": _chunk_plain, "rope": _rope_plain, "plan": _plan_plain}[c["op"]](s)
    if c["op"] == "decode":
        out = torch.empty_like(s["q"])
        s["cache"].skv_decode_attn_window(0, s["q"], s["table"], s["n"], out, s["work"], c["window"], c["sinks"])
        return out
    if c["op"] == "chunk":
        out = torch.empty_like(s["q"])
        s["cache"].skv_prefill_attn_window(0, s["q"], s["cu"], s["table"], s["n"], out, s["q_most"], c["window"], c["sinks"])
        return out
    if c["op"] == "rope":
        q = torch.empty(s["q"].shape, dtype=torch.bfloat16, device=s["q"].device)
        s["cache"].skv_rope_append(0, s["rope"], s["q"], q, s["k"], s["v"], s["pos"], s["slots"])
        return (q,) + s["held"]
    s["cache"].skv_plan_step(s["table"], s["n"], s["new"], s["free"], s["n_free"], s["slots"], s["cu"], s["n_out"], s["n_free_out"], positions=s["pos"])
    return _planned(s)


# ---- the definitions, in 64 bits -----------------------------------------------------------------------------------
def _exact_attention(s):
    """Sequence by sequence and head by head: every cached token that is held, a mask, exp, sums."""
    c, held, d = s["case"], s["held"], s["case"]["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    group, row = c["hq"] // c["hkv"], 0
    for b, (n, q) in enumerate(zip(*_lens(c))):
        if n == 0:
            row += q
            continue
        lo = max(0, n - q - c["window"] + 1)
        t = torch.tensor(list(range(min(c["sinks"], lo))) + list(range(lo, n)), device=out.device)
        slot = s["table"][b].long()[t // PAGE]
        if c["fp8"]:
            k = held[0][slot].permute(0, 1, 2, 4, 3, 5).flatten(2, 3).flatten(3)[torch.arange(len(t)), :, t % PAGE].double()
            v = held[1][slot].transpose(2, 3)[torch.arange(len(t)), :, t % PAGE].double()
            scale = held[2][slot][torch.arange(len(t)), :, :, t % PAGE].double()
            k, v = k * scale[:, :, :1], v * scale[:, :, 1:]
        else:
            both = held[0][slot].transpose(3, 4).flatten(4)[torch.arange(len(t)), :, :, t % PAGE].double()
            k, v = both[:, :, 0], both[:, :, 1]
        for r0 in range(0, q, 1024):
            pos = torch.arange(n - q + r0, n - q + min(q, r0 + 1024), device=out.device)[:, None]
            hidden = (t > pos) | ((t <= pos - c["window"]) & (t >= c["sinks"]))
            at = slice(row + r0, row + r0 + len(pos))
            for h in range(c["hq"]):
                x = s["q"][at, h].double() @ k[:, h // group].t() / math.sqrt(d)
                x[hidden] = -math.inf
                e = (x - x.max(1, keepdim=True).values).exp()
                out[at, h] = (e @ v[:, h // group]) / e.sum(1, keepdim=True)
        row += q
    return out


def _exact_rope(s):
    c, d = s["case"], s["case"]["d"]
    half = c["rotary"] // 2
    phase = torch.stack([s["pos"][a].double() * f for a, f in zip(_axis_of(c), s["freq"])], -1)[:, None]
    unit = torch.polar(torch.ones_like(phase), phase)
    i = torch.arange(half, device=phase.device)
    re, im = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + half)

    def turn(x):
        y = x.double().clone()
        z = torch.complex(y[..., re], y[..., im]) * unit
        y[..., re], y[..., im] = z.real, z.imag
        return y

    k = turn(s["k"])
    q, rows = turn(s["q"]), torch.stack((k, s["v"].double()), 2)           # [token][head][K|V][dim]
    pages = s["held"][0].shape[0]
    if c["fp8"]:                                          # (a code is a rounding, which has no value in 64 bits; its row's scale has)
        scales = torch.zeros((pages * PAGE, c["hkv"], 2), dtype=torch.float64, device=q.device)
        scales[s["slots"]] = rows.abs().amax(-1) / 448.0
        return [q, None, None, scales.view(pages, PAGE, c["hkv"], 2).permute(0, 2, 3, 1)]
    flat = torch.zeros((pages * PAGE, c["hkv"], 2, d), dtype=torch.float64, device=q.device)
    flat = flat.index_copy(0, s["slots"], rows).view(pages, PAGE, c["hkv"], 2, d // 8, 8)
    return [q, flat.permute(0, 2, 3, 4, 1, 5)]


def exact(case, seed):
    if case["op"] == "plan":
        return None                                      # whole numbers: they have to be the plain form's
    s = prepare(case, seed)
    return _exact_rope(s) if case["op"] == "rope" else _exact_attention(s)
