"""Plain statements of the page index, the selection of pages and attention over listed pages that the tests hold the
library to.  CPU tensors only; no code of the library's."""
import math

import numpy as np
import torch

PAGE = 16
TINY = 2.0 ** -100


def steps(x, largest):
    """Nearest whole numbers of 127ths of the largest, one fp32 operation at a time (numpy: every one of them IEEE)."""
    if not largest >= TINY:
        return np.zeros(x.shape, np.float32)
    return np.rint(x.astype(np.float32) * (np.float32(127.0) / np.float32(largest)))


def index_entry(k):
    """k [16][D] fp32: (codes [highest | lowest][D] int8, scale)."""
    k = k.float().numpy()
    if not np.isfinite(k).all():
        return torch.zeros(2, k.shape[1], dtype=torch.int8), math.inf
    ends = np.stack((k.max(0), k.min(0)))
    largest = np.abs(ends).max()
    codes = steps(ends, largest)
    return torch.from_numpy(codes.astype(np.int8)), float(np.float32(largest) / np.float32(127.0)) if largest >= TINY else 0.0


def scores(q, codes, scales):
    """q [rows][heads][D] of one run and kv head, codes [pages][2][D], scales [pages]: fp32 [pages]."""
    q = q.float().numpy()
    q = np.where(np.isfinite(q), q, np.float32(0))
    c = torch.from_numpy(steps(q, np.abs(q).max() if q.size else 0.0)).double().flatten(0, 1)
    hi, lo = codes[:, 0].double(), codes[:, 1].double()
    dot = (c.clamp(min=0) @ hi.T + c.clamp(max=0) @ lo.T).amax(0)
    got = dot.float() * scales.float()
    return torch.where(torch.isinf(scales), math.inf, got)


def page_list(score, p0, p1, top, first, last):
    """The list of a run at positions p0 to p1; score(page) for any page."""
    end = p1 // PAGE + 1
    begin, tail = min(first, end), max(min(first, end), p0 // PAGE - last + 1)
    between = sorted(range(begin, tail), key=lambda j: (-float(score[j]), j))[:top]
    return list(range(begin)) + sorted(between) + list(range(tail, end))


def attention(q, k, v, pos, pages, scale=None):
    """q [rows][heads of one kv head][D] at positions pos; k, v [n][D]; pages: a list.  Returns (out, sum of w |v|, largest
    scale sum |q k|) in 64 bits, as serving_reference.attention does; a page listed twice counts twice."""
    rows, heads, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    tokens = [t for p in pages for t in range(PAGE * p, PAGE * p + PAGE) if t < len(k)]
    t = torch.tensor(tokens, dtype=torch.long)
    seen = t[None] <= pos[:, None]
    t, seen = t[seen.any(0)], seen[:, seen.any(0)]              # (what no row sees may hold anything)
    kk, vv, q = k[t].double(), v[t].double(), q.double()
    x = torch.einsum("rhd,td->rht", q, kk) * scale
    x = x.masked_fill(~seen[:, None], -math.inf)
    top = x.amax(2, keepdim=True) if len(t) else torch.zeros(rows, heads, 1, dtype=torch.float64)
    e = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = e.sum(2, keepdim=True)
    w = e / torch.where(total == 0, 1.0, total)
    reach = (torch.einsum("rhd,td->rht", q.abs(), kk.abs()) * scale).masked_fill(~seen[:, None], 0.0)
    return (torch.einsum("rht,td->rhd", w, vv), torch.einsum("rht,td->rhd", w, vv.abs()),
            reach.amax(2, keepdim=True) if len(t) else torch.zeros(rows, heads, 1, dtype=torch.float64))
