"""The stored form of the cache in 8 bits, as include/pair.h words it, against the 64-bit
form."""
import os
import re

import numpy as np
import pytest

from oracle import rollout

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = {"i8": "PAIR_CACHE_I8", "e4m3": "PAIR_CACHE_E4M3"}
MOST = {"i8": 127.0, "e4m3": 448.0}


def header():
    """The header's text, without line breaks and comment stars."""
    text = open(os.path.join(ROOT, "include", "pair.h")).read()
    return re.sub(r"\s+(\*\s+)?", " ", text)


@pytest.mark.parametrize("fmt", sorted(NAMES))
def test_least_exponent_is_the_headers(fmt):
    """Rows whose largest entry is at the header's limit, one step of fp32 beside it, and
    at the codes around it, under every exponent: the byte is the least one with which the
    entry is below the limit, and no code is cut off."""
    limit = float(re.search(r"below ([\d.]+) 2\^\(b - 127\) for " + NAMES[fmt], header()).group(1))
    near = [np.float64(np.nextafter(np.float32(limit), np.float32(x))) for x in (0.0, 1e9)]
    tops = [limit, *near, MOST[fmt], MOST[fmt] / 2, limit / 2, near[0] / 2, limit - 1, limit + 1]
    for e in range(-60, 61):
        x = np.array([[t, -0.3 * t, 0.0] for t in tops]) * 2.0 ** e
        c, b = rollout.store_q8(x, fmt)
        least = [min(y for y in range(255) if t * 2.0 ** e < limit * 2.0 ** (y - 127))
                 for t in tops]
        assert b.tolist() == least
        y = x * 2.0 ** (127.0 - b[:, None])  # nothing is cut off: the largest code is nearest
        if fmt == "i8":
            assert (np.abs(c - y) <= 0.5).all()
        else:
            assert (np.abs(c - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10)).all()
        assert (np.abs(c) <= MOST[fmt]).all()


def test_errors_are_within_the_headers_bounds():
    """Entries from the row's largest down to 2^-40 of it, midpoints between codes among
    them: each is off by at most what the header says, and by all of it somewhere."""
    rng = np.random.default_rng(0)
    text = header()
    half = 2.0 ** int(re.search(r"at most 2\^(-\d+) 2\^\(b - 127\) for PAIR_CACHE_I8",
                                text).group(1))
    m = re.search(r"at most max\(2\^(-\d+) \|x\|, 2\^(-\d+) 2\^\(b - 127\)\) for PAIR_CACHE_E4M3",
                  text)
    part, step = (2.0 ** int(x) for x in m.groups())
    x = rng.choice([-1.0, 1.0], (400, 64)) * 2.0 ** -rng.uniform(0, 40, (400, 64))
    x[:200] = np.ldexp(rng.integers(1, 64, (200, 64)) / 2.0, -rng.integers(0, 24, (200, 64)))
    x *= 2.0 ** rng.integers(-30, 30, (400, 1))
    for fmt in sorted(NAMES):
        c, b = rollout.store_q8(x, fmt)
        unit = 2.0 ** (b - 127.0)[:, None] * np.ones_like(x)
        off = np.abs(rollout.values_q8(c, b) - x)
        bound = half * unit if fmt == "i8" else np.maximum(part * np.abs(x), step * unit)
        assert (off <= bound).all()
        assert off.max() > 0 and (off > 0.9 * bound).any()
    for row, back in (([1.0, 2.0 ** -18], [1.0, 0.0]),  # 1 is 256 2^-8: codes down to 2^-17
                      ([1.0, 2.0 ** -17], [1.0, 2.0 ** -17])):
        assert rollout.values_q8(*rollout.store_q8(np.array([row]), "e4m3"))[0].tolist() == back
