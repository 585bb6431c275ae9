"""A frequency's phase, 2^64 inv_freq / 2 pi modulo 2^64, over the whole range of frequencies that are taken, against integers of
600 bits; and the angles at far positions that come of it."""
import ctypes
import math
import random
from fractions import Fraction

import pytest
import torch


def inverse_arctan(x, one):
    """arctan(1 / x) in units of 1 / one, by its series."""
    term = total = one // x
    n, sign = 3, -1
    while term:
        term //= x * x
        total += sign * (term // n)
        n, sign = n + 2, -sign
    return total


ONE = 1 << 600
TWO_PI = Fraction(8 * (4 * inverse_arctan(5, ONE) - inverse_arctan(239, ONE)), ONE)        # Machin's formula


def turns(inv_freq):
    """The exact fraction of a turn per position, in [0, 1)."""
    x = Fraction(inv_freq) / TWO_PI
    return x - math.floor(x)


FREQS = [1e6, -1e6, 999983.3, 12345.678, 1.0, 0.5, -0.5, 2 * math.pi, math.pi, math.nextafter(math.pi, 4), 1e-9, 2.0 ** -60, 5e-324, 1e-300, 0.0, -0.0, 6.283185307179587e5]


def test_phase_of_a_frequency():
    from paper_2604_22782_b200 import build
    f = ctypes.CDLL(build.build_test_hooks()).skv_test_rope_phase
    f.argtypes, f.restype = [ctypes.c_double], ctypes.c_uint64
    g = random.Random(1)
    for x in FREQS + [g.uniform(-1e6, 1e6) for _ in range(2000)] + [10 ** g.uniform(-30, 6) for _ in range(2000)]:
        want = turns(x) * 2 ** 64
        off = (f(x) - want) % 2 ** 64
        assert min(off, 2 ** 64 - off) <= Fraction(1, 2) + Fraction(1, 2 ** 20), x              # rounded to nearest


@pytest.mark.gpu
@pytest.mark.parametrize("adjacent", [False, True])
def test_angles_of_large_frequencies_at_far_positions(adjacent):
    """Positions near 2^31 at which a frequency's angle is nearly a whole number of turns: the sine is as small as the angle, and shows
    its error to 2^-8 of it, beside fp32's 2^-20."""
    import paper_2604_22782_b200 as skv
    freqs = [1e6 / (1 + 0.37 * i) for i in range(32)]
    exact = [turns(x) for x in freqs]
    positions, which = [], []
    for i, t in enumerate(exact):
        step = round(t * 2 ** 64)
        near = sorted(range(2 ** 31 - 1 - 30000, 2 ** 31 - 1), key=lambda p: min(p * step % 2 ** 64, -p * step % 2 ** 64))[:4]
        positions += near + [-p for p in near]
        which += [i] * 8
    n = len(positions)
    rope = skv.SkvRope(freqs, adjacent_pairs=adjacent)
    cache = skv.SkvCache([0, 0], 1, 64, 16, 1, allocate=True)
    at = torch.arange(32)
    first, second = (2 * at, 2 * at + 1) if adjacent else (at, at + 32)
    q = torch.zeros(n, 1, 64, dtype=torch.bfloat16)
    q[:, 0, first] = 1.0
    out = torch.empty(n, 1, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    cache.skv_rope_append(1, rope, q.cuda(), out, None, None, pos, None)
    got = out.cpu().double()
    for row, (p, i) in enumerate(zip(positions, which)):
        t = p * exact[i]
        t -= math.floor(t)
        angle = float((t if t < Fraction(1, 2) else t - 1) * TWO_PI)
        for value, want in ((got[row, 0, first[i]], math.cos(angle)), (got[row, 0, second[i]], math.sin(angle))):
            assert abs(value.item() - want) <= abs(want) * 2 ** -8 + 2 ** -20, (freqs[i], p)
