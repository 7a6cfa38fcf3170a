"""Pins of the oracle's group normalization to the last bit of its statistics, and of the range of its
Swish (no GPU)."""

import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import core
from workloads import make_groupnorm
from workloads.generate import INT8, INT16


def _exact_norm(p, z, W):
    """The group normalization of one utterance in Python's integers, without the Swish and the output's clamp."""
    L, d = z.shape
    cg = d // p.n_groups
    out = np.empty((L, d), dtype=object)
    for g in range(p.n_groups):
        v = [int(a) for a in z[:, g * cg:(g + 1) * cg].ravel()]
        n, S = len(v), sum(v)
        mean = Fraction(S, n)
        dev = math.ceil(sum((a - mean) ** 2 for a in v))
        R = 2 ** 55 // math.isqrt((65536 * dev // n + p.eps) * 65536)
        mu = math.floor(65536 * mean + Fraction(1, 2))
        for c in range(g * cg, (g + 1) * cg):
            A = math.floor(Fraction(int(p.gn_mult[c]) * R, 2 ** (40 - W)))
            C = int(p.gn_bias[c]) - math.floor(Fraction(mu * A, 65536))
            for t in range(L):
                out[t, c] = math.floor(Fraction(int(z[t, c]) * A + C, 2 ** p.gn_shift) + Fraction(1, 2))
    return out


@pytest.mark.parametrize("tin", [INT8, INT16])
@pytest.mark.parametrize("seed,eps", [(0, 1), (1, 1), (2, 30000), (3, 2 ** 31 - 1)])
def test_groupnorm_keeps_every_bit_of_its_statistics(tin, seed, eps):
    """Multipliers so large beside the shift that one unit of the mean, the deviations or the root moves the
    outputs, of values whose variance is small and whose means have fractions of both signs."""
    rng = np.random.default_rng(seed)
    W, T, d, G = (8, 16)[tin], 5, 32, 4
    p = make_groupnorm(d, G, 6, tin, INT16, False, 1 / 32, 1 / 4096)
    p.gn_mult = rng.integers(1 << 22, 1 << 23, d).astype(np.int32)
    p.gn_bias, p.gn_shift, p.eps = np.zeros(d, dtype=np.int64), 8 + W, eps
    z = rng.integers(-2, 2, (1, T, d)).astype((np.int8, np.int16)[tin])
    want = _exact_norm(p, z[0], W)
    # each channel's bias moves its own values into the output's range, a few at a time
    for t in range(T):
        p.gn_bias = np.array([-int(h) << p.gn_shift for h in want[t]], dtype=np.int64)
        x = core.groupnorm(p, z, None)
        moved = np.clip(np.vectorize(lambda a, b: int(a) - int(b))(want, want[t]), -32767, 32767)
        assert np.array_equal(x[0], moved.astype(np.int16))


def test_groupnorm_swish_takes_values_held_to_int16():
    """Normalized values past the Swish's grid count as its ends: +-16 in steps of 16 / 32767, whose Swish
    the output grid (+-32) holds."""
    p = make_groupnorm(16, 1, 6, INT16, INT16, True, 1 / 4096, 1 / 1024)
    z = np.zeros((1, 3, 16), dtype=np.int16)  # so that h is the bias

    def of(h):
        p.gn_bias = np.full(16, h, dtype=np.int64) << p.gn_shift
        return core.groupnorm(p, z)

    top, low = of(32767), of(-32767)
    assert abs(int(top[0, 0, 0]) - 16 * 1024) <= 16 and (top == top[0, 0, 0]).all() and (low == low[0, 0, 0]).all()
    for h in (32768, 40000, 1 << 20):
        assert np.array_equal(of(h), top) and np.array_equal(of(-h), low)
