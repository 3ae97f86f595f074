"""Host-side argument checks of the rollout step's entry points (no GPU: what
is refused is refused before any device call), and the 64-bit forms' own pins."""
import ctypes
import os
import subprocess
import sys

import numpy as np

from oracle import rollout

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_validation_without_device():
    """In a child process with no visible device: the placeholder pointers must
    never reach a kernel, even if a check were to let a call through."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    code = ("import sys; sys.path.insert(0, %r); import tests.test_rollout_abi as t; "
            "from paper_2608_11368_gb300 import binding, build; build.build(); "
            "t._checks(binding)" % ROOT)
    res = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                         timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]


def _refusals(fn, good, bad):
    """fn(*good) passes the argument checks (and then finds no device), every
    change in `bad` gives its status."""
    assert fn(*good) not in (0, 1, 3), "the placeholder call stops at the device"
    for at, value, status in bad:
        args = list(good)
        args[at] = value
        assert fn(*args) == status, (fn, at, value, fn(*args))


def _checks(L):
    lib = L.lib()
    P, big = ctypes.c_void_p, P_BIG
    S = L.CacheStrides
    one, odd = P(1 << 20), P((1 << 20) + 8)
    good = [4, 16, 8, one, one, one, one, 32, one, 64, one, one, one, one, one, one, None, None]
    _refusals(lib.pair_pages_extend, good,
              [(0, 0, 1), (1, 0, 1), (2, 0, 1), (3, None, 1), (4, None, 1), (5, None, 1),
               (6, None, 1), (7, -1, 1), (8, None, 1), (9, 0, 1), (9, big, 1), (10, None, 1),
               (11, None, 1), (12, None, 1), (13, None, 1), (14, None, 1), (15, None, 1)])
    st = S(16 * 2 * 64, 2 * 64, 64)
    good = [8, 2, 64, L.PAIR_BF16, one, 128, 64, one, 128, 64, one, 9, 16, one, st, one, st, None,
            None]
    _refusals(lib.pair_cache_append, good,
              [(0, 0, 1), (0, big, 1), (1, 0, 1), (2, 0, 1), (2, 60, 1), (3, 7, 1), (4, None, 1),
               (4, odd, 1), (5, 129, 1), (6, 63, 1), (7, None, 1), (8, 4, 1), (10, None, 1),
               (11, 0, 1), (12, 0, 1), (13, odd, 1), (14, S(2048, 128, 60), 1), (15, None, 1),
               (16, S(2047, 128, 64), 1)])
    need = L.pair_attend_workspace_size(3, 4, 2, 64, L.PAIR_BF16)
    assert need > 0
    good = [8, 3, 4, 2, 64, L.PAIR_BF16, one, 256, 64, one, st, one, st, 9, 16, one, 5, one, one,
            0.125, 0, one, one, one, need, None, None]
    _refusals(lib.pair_attend_paged, good,
              [(0, 0, 1), (0, big, 1), (1, 0, 1), (2, 3, 1), (2, 1, 1), (3, 0, 1), (4, 96, 2),
               (4, 0, 2), (5, 9, 1), (6, None, 1), (6, odd, 1), (7, 255, 1), (9, None, 1),
               (10, S(2048, 4, 64), 1), (11, odd, 1), (13, 0, 1), (14, 0, 1), (15, None, 1),
               (16, 0, 1), (17, None, 1), (18, None, 1), (19, float("nan"), 1),
               (19, float("inf"), 1), (20, -1, 1), (21, None, 1), (21, odd, 1), (23, None, 3),
               (23, P((1 << 20) + 128), 3), (24, need - 1, 3)])
    for args in ((0, 4, 2, 64, 1), (1, 4, 3, 64, 1), (1, 4, 0, 64, 1), (1, 4, 2, 80, 1),
                 (1, 4, 2, 64, 5), (1, 2, 4, 64, 1)):
        assert L.pair_attend_workspace_size(*args) == 0
    good = [8, 3, 100, L.PAIR_F32, one, 100, one, 100, one, one, one, one, one, one, one, None,
            None]
    _refusals(lib.pair_verify_drafts, good,
              [(0, 0, 1), (0, big, 1), (1, 0, 1), (2, 0, 1), (2, (1 << 22) + 1, 1), (3, 2, 1),
               (4, None, 1), (5, 99, 1), (7, 99, 1), (8, None, 1), (9, None, 1), (10, None, 1),
               (11, None, 1), (12, None, 1), (14, None, 1)])


P_BIG = 2 ** 31


def test_status_strings_of_the_new_codes():
    from paper_2608_11368_gb300 import binding as B, build
    build.build()
    for code in (10, 11):
        assert B.pair_status_string(code) != "unknown status"
        assert B.STATUS_NAMES[code].startswith("PAIR_ERR_")


def test_attend_form_is_softmax_attention():
    """Contiguous pages, one chunk: the textbook expression."""
    rng = np.random.default_rng(0)
    n, m, Hq, Hkv, D, page = 3, 11, 4, 2, 8, 4
    q = rng.standard_normal((n, Hq, D))
    k, v = rng.standard_normal((3, page, Hkv, D)), rng.standard_normal((3, page, Hkv, D))
    out, lse, _, _ = rollout.attend_paged(q, k, v, np.arange(3)[None], [m], [0, n], 0.3)
    kk, vv = k.reshape(-1, Hkv, D)[:m], v.reshape(-1, Hkv, D)[:m]
    for h in range(Hq):
        s = 0.3 * q[:, h] @ kk[:, h // 2].T
        s[np.arange(m)[None] > np.arange(m - n, m)[:, None]] = -np.inf
        w = np.exp(s - s.max(1, keepdims=True))
        assert np.allclose(out[:, h], w / w.sum(1, keepdims=True) @ vv[:, h // 2], atol=1e-12)
        assert np.allclose(lse[:, h], np.log(np.exp(s).sum(1)), atol=1e-12)


def test_verify_form_emits_the_target():
    """Exact: summed over the drafter's draws and a fine grid of both random
    numbers, the first emitted token has the target's distribution."""
    p, q = np.array([0.5, 0.2, 0.3], np.float32), np.array([0.1, 0.6, 0.3], np.float32)
    N = 400
    grid = ((np.arange(N) + 0.5) / N).astype(np.float32)
    got = np.zeros(3)
    for y in range(3):
        for u in grid:
            o = rollout.verify_drafts(np.stack([p, p]), np.array([0, y]), [0, 2],
                                      np.array([u, 0], np.float32), np.array([0.5], np.float32),
                                      np.stack([q, q]))
            if o["n"][0] == 2:
                got[o["ids"][0]] += q[y] / N
            else:
                for ud in grid[::20]:
                    o = rollout.verify_drafts(np.stack([p, p]), np.array([0, y]), [0, 2],
                                              np.array([u, 0], np.float32), np.array([ud]),
                                              np.stack([q, q]))
                    got[o["ids"][0]] += q[y] / N / (N // 20)
    assert np.abs(got - p).max() <= 3.0 / N + 1.0 / (N // 20) * 0.5  # the grids' resolution


def test_pages_form_by_hand():
    o = rollout.pages_extend([3, 16], [1, 1], [2, 1], [7, 9], 2, np.array([[4, -1], [5, -1]]), 16, 4)
    assert o["table"].tolist() == [[4, -1], [5, 7]] and o["taken"] == 1 and not o["error"]
    assert o["slots"].tolist() == [4 * 16 + 3, 4 * 16 + 4, 7 * 16, -1]
    assert o["cu"].tolist() == [0, 2, 3] and o["kv_len"].tolist() == [5, 17]
