"""Limits of the rollout step's arguments (no GPU: refused before any device call)."""
import ctypes
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_requests_beyond_32_bit_indexes_are_refused():
    """In a child process without a device. With R near 2^31 a thread's run of
    requests would end at a negative index, and its requests be left out in
    silence."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    code = ("import sys; sys.path.insert(0, %r); import tests.test_rollout_limits as t; "
            "from paper_2608_11368_gb300 import binding, build; build.build(); "
            "t._checks(binding)" % ROOT)
    res = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                         timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]


def _checks(L):
    lib, S = L.lib(), L.CacheStrides
    one, invalid = ctypes.c_void_p(1 << 20), 1
    st = S(16 * 2 * 64, 2 * 64, 64)
    need = L.pair_attend_workspace_size(3, 4, 2, 64, L.PAIR_BF16)
    for R, ok in ((1 << 30, True), ((1 << 30) + 1, False), (2 ** 31 - 1, False)):
        got = lib.pair_pages_extend(R, 16, 8, one, one, one, one, 32, one, 64, one, one, one, one,
                                    one, one, None, None)
        assert (got != invalid) == ok
        got = lib.pair_attend_paged(8, R, 4, 2, 64, L.PAIR_BF16, one, 256, 64, one, st, one, st, 9,
                                    16, one, 5, one, one, 0.125, 0, one, one, one, need, None, None)
        assert (got != invalid) == ok
