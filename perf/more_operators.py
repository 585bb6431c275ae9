"""What is measured of sparse attention over selected pages: the index of the pages' keys, the selection of pages by a
cheap score, and attention over the selected pages (decode and chunk).

Each operator has a plain form in elementary torch operations and the call a user makes of the library.  Both work on the
same state: the page pool and the index are laid out as the library lays them out (plain tensors here), so neither side
converts anything that the other does not."""
import math

import torch

own = False

PAGE = 16
HEADER = 256            # bytes before the first page of a pool
TINY = 2.0 ** -100      # a largest element below this counts as none


# ---- cases -------------------------------------------------------------------------------------------------------
# Sequences hold lo to hi tokens before the call's new ones, which are q_lo to q_hi (decode: one each).
def _index(name, batch, hkv, d, lo, hi, q_lo, q_hi, fp8=False, decode=False):
    return {"name": name, "op": "index", "batch": batch, "hq": hkv, "hkv": hkv, "d": d, "lo": lo, "hi": hi, "q_lo": q_lo, "q_hi": q_hi,
            "fp8": fp8, "decode": decode}


def _select(name, batch, hq, hkv, d, lo, hi, top, first, last, q_lo=1, q_hi=1, run=0):
    return {"name": name, "op": "select", "batch": batch, "hq": hq, "hkv": hkv, "d": d, "lo": lo, "hi": hi, "q_lo": q_lo, "q_hi": q_hi,
            "decode": run == 0, "run": max(run, 1), "top": top, "first": first, "last": last, "fp8": False}


def _attend(name, batch, hq, hkv, d, lo, hi, top, first, last, q_lo=1, q_hi=1, run=0, fp8=False):
    return {"name": name, "op": "attend", "batch": batch, "hq": hq, "hkv": hkv, "d": d, "lo": lo, "hi": hi, "q_lo": q_lo, "q_hi": q_hi,
            "decode": run == 0, "run": max(run, 1), "top": top, "first": first, "last": last, "fp8": fp8}


def listed():
    return [
        # a decode step: one sequence in sixteen has just filled a page
        _index("index_64_step", 64, 8, 128, 4096, 16383, 1, 1, decode=True),
        # prompts in whole
        _index("index_8x4096", 8, 8, 128, 0, 0, 4096, 4096),
        # ragged chunks behind histories, FP8 pages
        _index("index_fp8_23_ragged", 23, 8, 128, 0, 5000, 1, 2000, fp8=True),
        # one user at long context: nothing but latency
        _select("select_1_32k", 1, 32, 8, 128, 32767, 32767, 112, 1, 15),
        # a full server
        _select("select_64_32k", 64, 32, 8, 128, 8191, 32767, 112, 1, 15),
        # two chunks of prompts behind long histories, 32 rows to a list
        _select("select_2x1024_run32", 2, 32, 8, 128, 30000, 30000, 112, 1, 13, 1024, 1024, 32),
        # one user's token: 2048 of 32768 tokens attended
        _attend("decode_1_128p", 1, 32, 8, 128, 32767, 32767, 112, 1, 15),
        # a mid-sized batch
        _attend("decode_32_128p", 32, 32, 8, 128, 16383, 32767, 112, 1, 15),
        # a full server on FP8 pages, twice as many pages
        _attend("decode_128_fp8_256p", 128, 32, 8, 128, 8191, 16383, 240, 1, 15, fp8=True),
        # short drafts of three query heads per kv head, head_dim 64, four rows to a list
        _attend("chunk_5_d64_run4", 5, 6, 2, 64, 2000, 2000, 60, 1, 4, 1, 30, 4),
        # two chunks of prompts behind long histories, 32 rows to a list
        _attend("chunk_2x1024_run32", 2, 32, 8, 128, 30000, 30000, 112, 1, 13, 1024, 1024, 32),
        # ragged chunks on FP8 pages
        _attend("chunk_4_fp8_run32", 4, 32, 8, 128, 12000, 16000, 112, 1, 13, 129, 256, 32, fp8=True),
    ]


HEADS = [(32, 8, 128), (32, 32, 128), (8, 1, 128), (4, 4, 128), (6, 2, 128), (8, 2, 128), (4, 2, 64), (6, 2, 64)]


def _log(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    op = rng.choice(["index", "select", "select chunk", "decode", "decode", "chunk", "chunk"])
    hq, hkv, d = rng.choice(HEADS)
    hi = _log(rng, 16, 32767)
    lo = rng.randint(0, hi)
    if op == "index":
        decode = rng.random() < 0.4
        q_hi = 1 if decode else _log(rng, 1, 4096)
        batch = _log(rng, 1, max(1, min(64, 1_000_000_000 // (hkv * d * (hi + q_hi)), 33_500_000 // (hkv * d * q_hi))))
        c = _index("", batch, hkv, d, lo, hi, rng.randint(1, q_hi), q_hi, fp8=rng.random() < 0.4, decode=decode)
        del c["name"]
        return c
    first, last, top = rng.choice([0, 1, 1, rng.randint(2, 6)]), rng.randint(1, 20), _log(rng, 1, 240)
    pages = min(first + last + top + 1, hi // PAGE + 1)
    if op == "select":
        batch = _log(rng, 1, max(1, min(64, 1_000_000_000 // (hkv * d * hi))))
        c = _select("", batch, hq, hkv, d, lo, hi, top, first, last)
    elif op == "decode":
        batch = _log(rng, 1, max(1, min(128, 268_000_000 // (hkv * d * pages * PAGE), 2_000_000_000 // (hkv * d * hi))))
        c = _attend("", batch, hq, hkv, d, lo, hi, top, first, last, fp8=rng.random() < 0.4)
    else:
        fp8 = op == "chunk" and rng.random() < 0.3
        run = rng.choice([1, 4, rng.randint(1, 16), 16 if hq // hkv > 4 else 32])
        q_hi = _log(rng, 1, 32 * run)
        most = min(2_000_000_000 // (hkv * d * (hi + q_hi)), 134_000_000 // (hq * q_hi * (pages * PAGE if op == "chunk" else hi // PAGE + 1)))
        batch = _log(rng, 1, max(1, min(8, most)))
        c = (_attend("", batch, hq, hkv, d, lo, hi, top, first, last, rng.randint(1, q_hi), q_hi, run, fp8) if op == "chunk" else
             _select("", batch, hq, hkv, d, lo, hi, top, first, last, rng.randint(1, q_hi), q_hi, run))
    del c["name"]
    return c


# ---- sizes that follow from a case ---------------------------------------------------------------------------------
def _spread(lo, hi, n, salt):
    """n whole numbers of [lo, hi], the first of them hi, the same ones for a case every time."""
    return [hi if i == 0 else lo + ((i + salt) * 2654435761 % 4294967296) * (hi - lo + 1) // 4294967296 for i in range(n)]


def _lens(c):
    """(cached tokens, new tokens) of every sequence, the new ones counted among the cached ones."""
    q = _spread(c["q_lo"], c["q_hi"], c["batch"], 1)
    return [x + y for x, y in zip(_spread(c["lo"], c["hi"], c["batch"], 7), q)], q


def _runs(c):
    """(sequence, first position, last position) of every list; a run that a sequence has no rows for has first > last."""
    got, per = [], -(-c["q_hi"] // c["run"])
    for b, (n, q) in enumerate(zip(*_lens(c))):
        for r in range(per):
            got.append((b, n - q + r * c["run"], n - q + min(q, (r + 1) * c["run"]) - 1))
    return got


def _width(c):
    """Entries of a list."""
    return min(c["top"] + c["first"] + c["last"] + (c["run"] + 14) // PAGE, max(-(-n // PAGE) for n in _lens(c)[0]))


def _candidates(c, p0):
    """Pages that are scored for a run that begins at position p0: [first, this)."""
    return max(p0 // PAGE - c["last"] + 1, c["first"])


def _listed_pages(c, p0, p1):
    cand = _candidates(c, p0) - c["first"]
    return p1 // PAGE + 1 - max(0, cand - c["top"])


def work(case):
    c = case
    n, q = _lens(c)
    if c["op"] == "index":
        pages = sum(x // PAGE - (x - y) // PAGE for x, y in zip(n, q))
        row = c["d"] + 4 if c["fp8"] else 2 * c["d"]
        return {"bytes": pages * c["hkv"] * (PAGE * row + 2 * c["d"] + 4) + 4 * pages + 8 * c["batch"], "flops": 2 * pages * c["hkv"] * PAGE * c["d"]}
    runs = [x for x in _runs(c) if x[1] <= x[2]]
    group = c["hq"] // c["hkv"]
    rows_bytes = sum(q) * c["hq"] * c["d"] * 2
    if c["op"] == "select":
        scored, most = 0, {}
        for b, p0, p1 in runs:
            cand = _candidates(c, p0) - c["first"]
            if cand > c["top"]:
                scored += cand * (p1 - p0 + 1)
                most[b] = max(most.get(b, 0), cand)
        listed_ = sum(_listed_pages(c, p0, p1) for _, p0, p1 in runs)
        return {"bytes": sum(most.values()) * (c["hkv"] * (2 * c["d"] + 4) + 4) + rows_bytes + 4 * c["hkv"] * (listed_ + len(runs)) + 8 * c["batch"],
                "flops": 2 * c["d"] * c["hq"] * scored}
    tokens, pairs = {}, 0
    for b, p0, p1 in runs:
        pages = _listed_pages(c, p0, p1)
        before = (pages - (p1 // PAGE - p0 // PAGE + 1)) * PAGE             # tokens of the pages before the first row's own
        pairs += sum(before + p % PAGE + 1 + (p // PAGE - p0 // PAGE) * PAGE for p in range(p0, p1 + 1))
        tokens[b] = tokens.get(b, 0) + before + p1 + 1 - p0 // PAGE * PAGE
    row = c["d"] + 4 if c["fp8"] else 2 * c["d"]
    held = sum(min(t, n[b]) for b, t in tokens.items())                     # (runs of a sequence share most of their pages)
    listed_ = sum(_listed_pages(c, p0, p1) for _, p0, p1 in runs)
    return {"bytes": held * c["hkv"] * 2 * row + 2 * rows_bytes + 4 * c["hkv"] * (listed_ + len(runs)) + 8 * c["batch"],
            "flops": 4 * c["d"] * group * c["hkv"] * pairs}


# ---- inputs --------------------------------------------------------------------------------------------------------
def _table(c, g, dev):
    """(page table, pages of the pool): pages in a random order."""
    n = torch.tensor(_lens(c)[0], device=dev)
    width = max(1, -(-int(n.max()) // PAGE))
    held = torch.arange(width, device=dev)[None] * PAGE < n[:, None]
    total = max(1, int(held.sum()))
    table = torch.full((len(n), width), -1, dtype=torch.int32, device=dev)
    table[held] = torch.randperm(total, generator=g, device=dev)[: int(held.sum())].to(torch.int32)
    return table, total


def _pool(c, pages, dev):
    """Bytes of a pool of one owner layer and what it holds, as views: bf16 [page][head][K|V][chunk of 8][token][8]; on FP8 pages
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


def _fill(c, held, g, dev):
    """Keys and values of every slot: what projections of normalised activations look like."""
    if not c["fp8"]:
        held[0].normal_(generator=g)
        return
    pages, h, d = held[1].shape[0], c["hkv"], c["d"]
    u = torch.uint8
    for i in range(0, pages, 4096):                              # (in pieces: the largest pool is some gigabytes)
        at = slice(i, min(pages, i + 4096))
        both = torch.randn((at.stop - i, 2, h, PAGE, d), generator=g, device=dev)
        amax = both.abs().amax(-1, keepdim=True)
        codes = (both * (448.0 / amax)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(u)
        held[0].view(u)[at] = codes[:, 0].reshape(-1, h, 2, 8, d // 16, 16).transpose(3, 4)
        held[1].view(u)[at] = codes[:, 1].transpose(2, 3)
        held[2][at] = (amax[..., 0] / 448.0).transpose(1, 2)


def _index_views(c, memory, pages):
    """Codes [page][head][highest|lowest][dim] and scales [page][head] of an index of one owner layer."""
    h, d = c["hkv"], c["d"]
    n = pages * h * 2 * d
    return memory[:n].view(torch.int8).view(pages, h, 2, d), memory[-(-n // 256) * 256:][:4 * pages * h].view(torch.float32).view(pages, h)


def _index_bytes(c, pages):
    up = lambda x: -(-x // 256) * 256  # noqa: E731
    return up(pages * c["hkv"] * 2 * c["d"]) + up(pages * c["hkv"] * 4)


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    s = {"case": c}
    s["table"], pages = _table(c, g, dev)
    s["pool"], s["held"] = _pool(c, pages, dev)
    n, q = _lens(c)
    s["n"] = torch.tensor(n, dtype=torch.int32, device=dev)
    s["cu"] = torch.tensor([0] + torch.tensor(q).cumsum(0).tolist(), dtype=torch.int32, device=dev)
    s["q_most"] = max(q)
    if own:
        import paper_2604_22782_b200 as skv
        s["cache"] = skv.SkvCache([0], c["hkv"], c["d"], PAGE, pages, device_pool=s["pool"], fp8=c["fp8"])
    if c["op"] != "attend":
        memory = torch.zeros(_index_bytes(c, pages), dtype=torch.uint8, device=dev)
        s["codes"], s["scales"] = _index_views(c, memory, pages)
        if own:
            s["cache"].skv_set_page_index(memory)
    if c["op"] == "index":
        _fill(c, s["held"], g, dev)
        return s
    s["q"] = torch.randn((sum(q), c["hq"], c["d"]), generator=g, device=dev).to(torch.bfloat16)
    runs = _runs(c)
    s["seq"], s["p0"], s["p1"] = (torch.tensor([x[i] for x in runs], device=dev) for i in range(3))
    lists, heads = len(runs), c["hkv"]
    s["lists"] = torch.full((lists, heads, _width(c)), -1, dtype=torch.int32, device=dev)
    s["counts"] = torch.zeros((lists, heads), dtype=torch.int32, device=dev)
    if c["op"] == "select":
        # highest and lowest key of a page around a mean of its own; pages that matter more and less
        mid = torch.randn((pages, heads, c["d"]), generator=g, device=dev) * 24
        half = torch.randn((pages, heads, c["d"]), generator=g, device=dev).abs() * 8 + 30
        s["codes"][:, :, 0] = (mid + half).round().clamp(-127, 127).to(torch.int8)
        s["codes"][:, :, 1] = (mid - half).round().clamp(-127, 127).to(torch.int8)
        s["scales"].copy_(torch.randn((pages, heads), generator=g, device=dev).mul(0.1).exp() * 0.03)
        return s
    _fill(c, s["held"], g, dev)
    for i in range(0, lists, 256):
        at = slice(i, i + 256)
        score = torch.rand((len(s["seq"][at]), heads, s["table"].shape[1]), generator=g, device=dev)
        s["lists"][at], s["counts"][at] = _chosen(c, score, s["p0"][at], s["p1"][at], s["lists"].shape[2])
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------
def _chosen(c, score, p0, p1, width):
    """Lists [list][head][width] of the pages to attend, ascending, -1 behind the last, and their number: the first pages, the last
    ones and the `top` others with the highest score, of two equal ones the lower."""
    j = torch.arange(score.shape[-1], device=score.device)
    own_page, end = (p0 // PAGE)[:, None, None], (p1 // PAGE)[:, None, None]
    there = (j <= end) & (p0 <= p1)[:, None, None]
    scored = there & (j >= c["first"]) & (j <= own_page - c["last"])
    order = torch.where(scored, score, -math.inf).sort(dim=-1, descending=True, stable=True).indices
    best = torch.zeros_like(score, dtype=torch.bool).scatter_(-1, order[..., :c["top"]], True) & scored
    take = (best | (there & ~scored)).expand(score.shape)
    counts = take.sum(-1)
    at = torch.where(take, take.cumsum(-1) - 1, width)                      # (a place behind the list for those not taken)
    lists = torch.full(score.shape[:-1] + (width + 1,), -1, dtype=torch.int64, device=score.device)
    lists.scatter_(-1, at.clamp(max=width), j.expand(score.shape))
    lists[..., width] = -1
    return lists[..., :width].to(torch.int32), counts.to(torch.int32)


def _steps(x, largest):
    """Whole steps of 1/127 of the largest; none where that is next to nothing."""
    some = largest >= TINY
    return torch.where(some, torch.round(x * (torch.full_like(largest, 127.0) / torch.where(some, largest, torch.ones_like(largest)))), torch.zeros_like(x))


def _index_plain(s):
    c, held, dev = s["case"], s["held"], s["n"].device
    n, cu = s["n"].long(), s["cu"].long()
    j = torch.arange(s["table"].shape[1], device=dev)[None]
    full = (j < (n // PAGE)[:, None]) & (j >= ((n - cu[1:] + cu[:-1]) // PAGE)[:, None])
    ids = s["table"][full].long()
    for i in range(0, len(ids), 4096):
        p = ids[i:i + 4096]
        if c["fp8"]:
            k = held[0].view(torch.uint8)[p].transpose(3, 4).reshape(len(p), c["hkv"], PAGE, c["d"]).view(torch.float8_e4m3fn).float() * held[2][p][:, :, 0, :, None]
        else:
            k = held[0][p, :, 0].float().transpose(2, 3).reshape(len(p), c["hkv"], PAGE, c["d"])
        ends = torch.stack((k.amax(2), k.amin(2)), 2)                       # [page][head][highest|lowest][dim]
        largest = ends.abs().amax((2, 3), keepdim=True)
        s["codes"][p] = _steps(ends, largest).to(torch.int8)
        s["scales"][p] = torch.where(largest >= TINY, largest / torch.full_like(largest, 127.0), torch.zeros_like(largest))[..., 0, 0]
    return s["codes"], s["scales"]


def _select_plain(s):
    c, dev = s["case"], s["q"].device
    heads, group, d, run = c["hkv"], c["hq"] // c["hkv"], c["d"], c["run"]
    per = -(-s["q_most"] // run)
    for b in range(c["batch"]):
        lists = slice(b * per, (b + 1) * per)
        rows = s["q"][int(s["cu_host"][b]):int(s["cu_host"][b + 1])].float()
        rows = torch.nn.functional.pad(rows, (0, 0, 0, 0, 0, per * run - len(rows)))
        rows = rows.view(per, run, heads, group, d).permute(0, 2, 1, 3, 4).flatten(2, 3)       # [list][head][row and query head][dim]
        codes = _steps(rows, rows.abs().amax((2, 3), keepdim=True))
        both = torch.cat((codes.clamp(min=0), codes.clamp(max=0)), -1)
        ids = s["table"][b].clamp(min=0).long()
        ends = s["codes"][ids].float().flatten(2).permute(1, 2, 0)                            # [head][highest and lowest][page]
        score = torch.matmul(both, ends).amax(2) * s["scales"][ids].t()                       # (whole numbers below 2^24 until here)
        s["lists"][lists], s["counts"][lists] = _chosen(c, score, s["p0"][lists], s["p1"][lists], s["lists"].shape[2])
    return s["lists"], s["counts"]


def _keys_and_values(s, lists, seq):
    """K and V in 32 bits of listed pages [list][head][width]: [list][head][tokens][dim]."""
    c, held = s["case"], s["held"]
    page = s["table"][seq].long().gather(1, lists.clamp(min=0).long().flatten(1)).clamp(min=0).view(lists.shape)
    head = torch.arange(c["hkv"], device=page.device)[None, :, None]
    if c["fp8"]:
        scale = held[2][page, head]
        k = held[0].view(torch.uint8)[page, head].transpose(4, 5).reshape(page.shape + (PAGE, c["d"])).view(torch.float8_e4m3fn).float() * scale[..., 0, :, None]
        v = held[1].view(torch.uint8)[page, head].view(torch.float8_e4m3fn).float().transpose(3, 4) * scale[..., 1, :, None]
    else:
        k, v = held[0][page, head].float().transpose(4, 5).flatten(5).unbind(3)
    return k.flatten(2, 3), v.flatten(2, 3)


def _attend_plain(s):
    c, dev = s["case"], s["q"].device
    heads, group, d, run = c["hkv"], c["hq"] // c["hkv"], c["d"], c["run"]
    out = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device=dev)
    cu, piece = s["cu"].long(), max(1, 2_000_000_000 // (heads * d * s["lists"].shape[2] * PAGE * 8))
    for i in range(0, len(s["seq"]), piece):
        at = slice(i, i + piece)
        lists, seq, p0, p1 = s["lists"][at], s["seq"][at], s["p0"][at], s["p1"][at]
        k, v = _keys_and_values(s, lists, seq)
        pos = p0[:, None] + torch.arange(run, device=dev)                                     # [list][row]
        row = cu[seq + 1][:, None] - s["n"][seq].long()[:, None] + pos
        there = pos <= p1[:, None]
        q = s["q"].float()[torch.where(there, row, 0)].view(len(seq), run, heads, group, d).permute(0, 2, 1, 3, 4)
        x = torch.matmul(q.flatten(2, 3), k.transpose(2, 3)).view(len(seq), heads, run, group, -1) / math.sqrt(d)
        token = (lists[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(2)
        seen = ((token >= 0) & (lists >= 0).repeat_interleave(PAGE, 2))[:, :, None] & (token[:, :, None] <= pos[:, None, :, None])
        x = x.masked_fill(~seen[:, :, :, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        e = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
        total = e.sum(-1, keepdim=True)
        o = torch.matmul((e / torch.where(total > 0, total, torch.ones_like(total))).flatten(2, 3), v).view(q.shape)
        out[row[there]] = o.permute(0, 2, 1, 3, 4).flatten(2, 3)[there].to(torch.bfloat16)
    return out


def run(state):
    s, c = state, state["case"]
    if not own:
        if "cu_host" not in s:
            s["cu_host"] = [0] + torch.tensor(_lens(c)[1]).cumsum(0).tolist()
        return {"index": _index_plain, "select": _select_plain, "attend": _attend_plain}[c["op"]](s)
    if c["op"] == "index":
        if c["decode"]:
            s["cache"].skv_index_pages(0, s["table"], s["n"])
        else:
            s["cache"].skv_index_pages(0, s["table"], s["n"], cu_q_lens=s["cu"], max_q_len=s["q_most"])
        return s["codes"], s["scales"]
    if c["op"] == "select":
        if c["decode"]:
            s["cache"].skv_select_pages(0, s["q"], s["table"], s["n"], s["lists"], s["counts"], c["top"], c["first"], c["last"])
        else:
            s["cache"].skv_select_pages(0, s["q"], s["table"], s["n"], s["lists"], s["counts"], c["top"], c["first"], c["last"],
                                        cu_q_lens=s["cu"], max_q_len=s["q_most"], run=c["run"])
        return s["lists"], s["counts"]
    out = torch.empty_like(s["q"])
    if c["decode"]:
        s["cache"].skv_decode_attn_pages(0, s["q"], s["table"], s["n"], s["lists"], s["counts"], out)
    else:
        s["cache"].skv_prefill_attn_pages(0, s["q"], s["cu"], s["table"], s["n"], s["lists"], s["counts"], out, s["q_most"], run=c["run"])
    return out


# ---- the definitions, in 64 bits -----------------------------------------------------------------------------------
def _exact_scales(s):
    """The scale of every page that the call's tokens complete: a 127th of its largest key.  (The codes are roundings.)"""
    c, held = s["case"], s["held"]
    want = torch.zeros(s["scales"].shape, dtype=torch.float64, device=s["scales"].device)
    for b, (n, q) in enumerate(zip(*_lens(c))):
        for i in range((n - q) // PAGE, n // PAGE, 1024):
            page = s["table"][b, i:min(n // PAGE, i + 1024)].long()
            if c["fp8"]:
                k = held[0][page].double().permute(0, 1, 2, 4, 3, 5).reshape(len(page), c["hkv"], PAGE, -1)
                k = k * held[2][page, :, 0].double()[..., None]
            else:
                k = held[0][page, :, 0].double()
            want[page] = k.flatten(2).abs().max(2).values / 127.0
    return want


def _exact_attention(s):
    """List by list and head by head: the tokens of its pages, a mask, exp, sums."""
    c, held, d = s["case"], s["held"], s["case"]["d"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    group = c["hq"] // c["hkv"]
    n, new = _lens(c)
    start = [sum(new[:b]) for b in range(len(new))]
    lists = s["lists"].tolist()
    for i, (b, p0, p1) in enumerate(_runs(c)):
        if p0 > p1:
            continue
        pos = torch.arange(p0, p1 + 1, device=out.device)
        rows = slice(start[b] + p0 - (n[b] - new[b]), start[b] + p1 + 1 - (n[b] - new[b]))
        for h in range(c["hkv"]):
            pages = torch.tensor([p for p in lists[i][h] if p >= 0], device=out.device)
            where = s["table"][b].long()[pages]
            if c["fp8"]:
                scale = held[2][where, h].double()
                k = held[0][where, h].double().permute(0, 1, 3, 2, 4).reshape(len(pages), PAGE, d) * scale[:, 0, :, None]
                v = held[1][where, h].double().permute(0, 2, 1) * scale[:, 1, :, None]
            else:
                both = held[0][where, h].double().permute(1, 0, 3, 2, 4)
                k, v = both[0].reshape(-1, PAGE, d), both[1].reshape(-1, PAGE, d)
            token = (pages[:, None] * PAGE + torch.arange(PAGE, device=out.device)).flatten()
            hidden = token[None] > pos[:, None]
            for m in range(h * group, (h + 1) * group):
                x = s["q"][rows, m].double() @ k.reshape(-1, d).t() / math.sqrt(d)
                x[hidden] = -math.inf
                e = (x - x.max(1, keepdim=True).values).exp()
                out[rows, m] = (e @ v.reshape(-1, d)) / e.sum(1, keepdim=True)
    return out


def exact(case, seed):
    if case["op"] == "select":
        return None                                      # whole numbers: they have to be the plain form's
    s = prepare(case, seed)
    return _exact_attention(s) if case["op"] == "attend" else [None, _exact_scales(s)]
