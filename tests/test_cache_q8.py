"""The cache in 8 bits, without a GPU: the 64-bit form's own pins, and what the entry
points refuse before any device call."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import rollout

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("fmt,most", [("i8", 127.0), ("e4m3", 448.0)])
def test_stored_form(fmt, most):
    """The least exponent with which nothing is cut off, nearest codes, and
    powers of two that move the exponent alone."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 16)) * np.exp(3 * rng.standard_normal((400, 1)))
    c, b = rollout.store_q8(x, fmt)
    assert np.abs(c).max() == most and (np.abs(c).max(-1) > most / 2 - 8).all()
    v = rollout.values_q8(c, b)
    s = 2.0 ** (b - 127.0)[:, None]
    if fmt == "i8":
        assert (c == np.rint(c)).all() and (np.abs(v - x) <= 0.5 * s).all()
    else:  # half a step: 2^-4 of the value, 2^-10 below the normal codes
        assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, s * 2.0 ** -10)).all()
    c2, b2 = rollout.store_q8(x * 2.0 ** 40, fmt)
    assert (c2 == c).all() and (b2 == b + 40).all()
    again, same = rollout.store_q8(v, fmt)
    assert (rollout.values_q8(again, same) == v).all()


def test_stored_form_by_hand():
    near = np.nextafter(127.5, 0)
    for row, codes, b in (([127.0, 0.5], [127, 0], 127), ([127.5, 1.5], [64, 1], 128),
                          ([near, -1.5], [127, -2], 127), ([0.0, -0.0], [0, 0], 0),
                          ([2.0 ** -127, 2.0 ** -128], [1, 0], 0),
                          ([np.inf, 1.0], [0, 0], 255), ([np.nan, 1.0], [0, 0], 255)):
        c, e = rollout.store_q8(np.array([row]), "i8")
        assert c[0].tolist() == codes and e[0] == b
    for row, codes, b in (([448.0, 17.0], [448, 16], 127), ([463.9, 0.001], [448, 2.0 ** -9], 127),
                          ([464.0, 1.0], [224, 0.5], 128), ([480.0, 1.0], [240, 0.5], 128),
                          ([19.0, 1.0], [320, 16], 123)):
        c, e = rollout.store_q8(np.array([row]), "e4m3")
        assert c[0].tolist() == codes and e[0] == b
    assert np.isnan(rollout.values_q8(np.array([[0.0]]), np.array([255]))).all()


def test_host_validation_without_device():
    """In a child process with no visible device: the placeholder pointers must
    never reach a kernel, even if a check were to let a call through."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    code = ("import sys; sys.path.insert(0, %r); import tests.test_cache_q8 as t; "
            "from paper_2608_11368_gb300 import binding, build; build.build(); "
            "t._checks(binding)" % ROOT)
    res = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                         timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]


def _checks(L):
    lib, S = L.lib(), L.CacheStrides
    P, big = ctypes.c_void_p, 2 ** 31
    one, odd = 1 << 20, (1 << 20) + 8
    st, byte = S(16 * 2 * 64, 2 * 64, 64), S(33, 2, 1)

    def cache(codes=one, at=st, exps=one, exps_at=byte):
        return L.CacheQ8(codes, at, exps, exps_at)

    def refusals(fn, good, bad):
        assert fn(*good) not in (0, 1, 3), "the placeholder call stops at the device"
        for at, value, status in bad:
            args = list(good)
            args[at] = value
            assert fn(*args) == status, (fn, at, value, fn(*args))

    caches = [(cache(codes=None), 1), (cache(codes=odd), 1), (cache(exps=None), 1),
              (cache(at=S(2048 + 8, 128, 64)), 1), (cache(at=S(2048, 128, 72)), 1),
              (cache(at=S(2048, 136, 64)), 1)]
    p = P(one)
    good = [8, 2, 64, L.PAIR_BF16, p, 128, 64, p, 128, 64, p, 9, 16, 0, cache(), cache(), None,
            None]
    refusals(lib.pair_cache_append_q8, good,
             [(0, 0, 1), (0, big, 1), (1, 0, 1), (2, 0, 1), (2, 8, 1), (2, 72, 1), (2, 272, 1),
              (3, 7, 1), (4, None, 1), (4, P(odd), 1), (5, 129, 1), (6, 63, 1), (7, None, 1),
              (8, 4, 1), (10, None, 1), (11, 0, 1), (12, 0, 1), (13, 2, 1), (13, -1, 1)]
             + [(x, c, s) for x in (14, 15) for c, s in caches])
    good = [8, 2, 64, p, 9, 16, 1, cache(), cache(), L.PAIR_F32, p, 128, 64, p, 128, 64, None, None]
    refusals(lib.pair_cache_read_q8, good,
             [(0, 0, 1), (0, big, 1), (1, 0, 1), (2, 24, 1), (3, None, 1), (4, 0, 1), (5, 0, 1),
              (6, 2, 1), (9, 2, 1), (10, None, 1), (10, P(odd), 1), (11, 130, 1), (13, None, 1),
              (15, 66, 1)] + [(x, c, s) for x in (7, 8) for c, s in caches])
    need = L.pair_attend_workspace_size(3, 4, 2, 64, L.PAIR_BF16)
    good = [8, 3, 4, 2, 64, L.PAIR_BF16, p, 256, 64, 0, cache(), cache(), 9, 16, p, 5, p, p, 0.125,
            0, p, p, p, need, None, None]
    refusals(lib.pair_attend_paged_q8, good,
             [(0, 0, 1), (0, big, 1), (1, 0, 1), (1, (1 << 30) + 1, 1), (2, 3, 1), (2, 1, 1),
              (3, 0, 1), (4, 96, 2), (4, 0, 2), (5, 9, 1), (6, None, 1), (6, P(odd), 1),
              (7, 255, 1), (9, 2, 1), (9, -1, 1), (12, 0, 1), (13, 0, 1), (14, None, 1),
              (15, 0, 1), (16, None, 1), (17, None, 1), (18, float("nan"), 1),
              (18, float("inf"), 1), (19, -1, 1), (20, None, 1), (20, P(odd), 1), (22, None, 3),
              (22, P(one + 128), 3), (23, need - 1, 3)]
             + [(x, c, s) for x in (10, 11) for c, s in caches])
    # Strides over a single entry are not looked at: one token, one head, one page.
    lone = cache(at=S(3, 5, 7), exps_at=S(0, 0, 0))
    for T, H, pages, page, ok in ((1, 1, 1, 1, True), (2, 1, 1, 1, False), (1, 2, 1, 1, False),
                                  (1, 1, 2, 1, False), (1, 1, 1, 2, False)):
        need = L.pair_attend_workspace_size(1, 1, 1, 64, L.PAIR_BF16)
        for got in (lib.pair_cache_append_q8(T, H, 64, L.PAIR_BF16, p, 3, 5, p, 7, 9, p, pages,
                                             page, 0, lone, lone, None, None),
                    lib.pair_cache_read_q8(T, H, 64, p, pages, page, 0, lone, lone, L.PAIR_BF16, p,
                                           3, 5, p, 7, 9, None, None),
                    lib.pair_attend_paged_q8(T, 1, H, H, 64, L.PAIR_BF16, p, 3, 5, 0, lone, lone,
                                             pages, page, p, 1, p, p, 0.1, 0, p, p, p, need, None,
                                             None)):
            assert (got != 1) == ok


def test_binding_refuses_tensors_of_the_host():
    import torch
    from paper_2608_11368_gb300 import binding as B
    k = torch.zeros((1, 1, 64))
    c, e = torch.zeros((1, 1, 1, 64), dtype=torch.int8), torch.zeros((1, 1, 1), dtype=torch.uint8)
    slots = torch.zeros(1, dtype=torch.int64)
    for call in (lambda: B.pair_cache_append_q8(k, k, slots, c, e, c, e),
                 lambda: B.pair_cache_read_q8(slots, c, e, c, e),
                 lambda: B.pair_attend_paged_q8(k, c, e, c, e, slots[None], slots, slots)):
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            call()
