"""Plain 64-bit statements of the serving-step operators (windowed attention, rotary embedding, a step's tables) that
the tests hold the library to, and the set-up they share.  CPU tensors only; no code of the library's."""
import math

import torch

PAGE = 16


def sees(pos, t, window, sinks):
    """Whether the row at position pos attends token t."""
    return t <= pos and (t > pos - window or t < sinks)


def attention(q, k, v, pos, window, sinks, scale=None):
    """One sequence: q [rows][Hq][D] at positions pos [rows]; k, v [n][Hkv][D].  Returns (out, sum of w |v|, largest
    scale sum |q k| of a row) in 64 bits: the latter two are what rounding errors are measured by."""
    rows, hq, d = q.shape
    n, hkv, _ = k.shape
    out, size, reach = torch.zeros(rows, hq, d, dtype=torch.float64), torch.zeros(rows, hq, d, dtype=torch.float64), torch.zeros(rows, hq, 1, dtype=torch.float64)
    if n == 0 or rows == 0:
        return out, size, reach
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    t, p = torch.arange(n)[None], pos[:, None]
    seen = (t <= p) & ((t > p - window) | (t < sinks))
    # tokens that no row sees may hold anything: they are not part of the definition
    any_row = seen.any(0)
    q = q.double()
    k = torch.where(any_row[:, None, None], k.double(), 0.0)
    v = torch.where(any_row[:, None, None], v.double(), 0.0)
    for h in range(hq):
        kh, vh = k[:, h // (hq // hkv)], v[:, h // (hq // hkv)]
        x = (q[:, h] @ kh.T * scale).masked_fill(~seen, -math.inf)
        w = torch.softmax(x, 1)
        out[:, h], size[:, h] = w @ vh, w @ vh.abs()
        reach[:, h, 0] = (q[:, h].abs() @ kh.abs().T * scale).masked_fill(~seen, 0.0).amax(1)
    return out, size, reach


def attention_tolerance(out, size, reach, n, fp8, v_max=0.0):
    """|error| of an output element.  Roundings: the result to bf16 (half a step, 2^-8 of it), the probabilities to
    bf16 (2^-8 each, so 2^-8 sum w |v|) or, on FP8 pages, to f16 (2^-11, and half the smallest step, 2^-25, of values up to
    the largest V times two where they are tiny).  Scores: 128 fp32 additions of products, each off by 2^-23 at most, or on
    FP8 pages the query rounded to f16 (2^-11 of every product); a score off by e moves every weight by e and their sum
    by e: 2 e sum w |v|.  exp2 and the fp32 sums: well below 2^-16."""
    if fp8:
        return out.abs() * 2 ** -8 + size * (2 ** -11 + 2 * 2 ** -11 * reach + 2 ** -15) + n * 2 ** -24 * v_max
    return out.abs() * 2 ** -8 + size * (2 ** -8 + 2 * 128 * 2 ** -23 * reach + 2 ** -15)


def angles(positions, inv_freq, axis):
    """[n][frequencies] in 64 bits; positions [axes][n]."""
    return positions.double()[torch.tensor(axis)].T * torch.tensor(inv_freq, dtype=torch.float64)


def rope(x, angle, adjacent):
    """[n][heads][D] turned in 64 bits; the second result is what an fp32 evaluation's error is measured by."""
    half = angle.shape[1]
    y, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64)
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    u, w = x.double()[..., a], x.double()[..., b]
    y[..., a], y[..., b] = u * c - w * s, w * c + u * s
    size[..., a] = size[..., b] = u.abs() + w.abs()
    return y, size


def rope_tolerance(y, size):
    """One rounding to bf16 (2^-8 of the value), and fp32: the angle to 2^-24 of half a turn, cos and sin to a few ulp,
    two products and a sum: below 2^-20 of |x1| + |x2|."""
    return y.abs() * 2 ** -8 + size * 2 ** -20


def plan_step(table, lens, new, free, n_free, max_tokens):
    """Request by request.  Returns (table, slots, positions, cu, lens, pages left, refused requests)."""
    table = [list(r) for r in table]
    slots, positions, cu, out, refused = [], [], [0], [], []
    stack, want_pages, want_tokens = list(free[:max(0, min(n_free, len(free)))]), 0, 0
    n_free = len(stack)
    for b, (n, a) in enumerate(zip(lens, new)):
        n, a = max(n, 0), max(a, 0)
        need = -(-(n + a) // PAGE) - -(-n // PAGE)
        want_pages += need
        want_tokens += a
        ok = (need == 0 or want_pages <= n_free) and want_tokens <= max_tokens and n + a <= len(table[b]) * PAGE
        if not ok:
            if a:
                refused.append(b)
            a = need = 0
        for k in range(need):
            table[b][-(-n // PAGE) + k] = stack.pop()
        for t in range(n, n + a):
            slots.append(table[b][t // PAGE] * PAGE + t % PAGE)
            positions.append(t)
        cu.append(cu[-1] + a)
        out.append(n + a)
    return table, slots, positions, cu, out, len(stack), refused


def paged(lens, g, spare=0, width=None):
    """A page table of random pages for sequences of these lengths, and the pages in the pool."""
    pages = [-(-n // PAGE) for n in lens]
    total = max(1, sum(pages) + spare)
    order = torch.randperm(total, generator=g).tolist()
    width = width or max(1, max(pages))
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    for b, p in enumerate(pages):
        for j in range(p):
            table[b, j] = order.pop()
    return table, total


def slots_of(table, b, t):
    """Slot of every token of t in sequence b."""
    return table[b].long()[t // PAGE] * PAGE + t % PAGE
