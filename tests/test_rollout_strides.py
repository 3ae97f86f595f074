"""Strides over a single entry say nothing: a view of one row, one head, one page or
pages of one token is taken whatever they are."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from tests.test_gpu_attend import build, check

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_host_checks_leave_them_out():
    """In a child process without a device, where a call that passes the checks
    stops."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="")
    code = ("import sys; sys.path.insert(0, %r); import tests.test_rollout_strides as t; "
            "from paper_2608_11368_gb300 import binding, build; build.build(); "
            "t._checks(binding)" % ROOT)
    res = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True,
                         timeout=600)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-2000:]


def _checks(L):
    lib, S = L.lib(), L.CacheStrides
    one = ctypes.c_void_p(1 << 20)
    invalid = 1
    # One token, one head, one page: every stride is odd.
    st = S(3, 5, 7)
    need = L.pair_attend_workspace_size(1, 1, 1, 64, L.PAIR_BF16)
    for T, H, pages, page, ok in ((1, 1, 1, 1, True), (2, 1, 1, 1, False), (1, 2, 1, 1, False),
                                  (1, 1, 2, 1, False), (1, 1, 1, 2, False)):
        got = lib.pair_cache_append(T, H, 64, L.PAIR_BF16, one, 3, 5, one, 7, 9, one, pages, page,
                                    one, st, one, st, None, None)
        assert (got != invalid) == ok
        got = lib.pair_attend_paged(T, 1, H, H, 64, L.PAIR_BF16, one, 3, 5, one, st, one, st, pages,
                                    page, one, 1, one, one, 0.1, 0, one, one, one, need, None, None)
        assert (got != invalid) == ok
    for T, ok in ((1, True), (2, False)):
        got = lib.pair_verify_drafts(T, 1, 100, L.PAIR_F32, one, 1, one, 1, one, one, one, one, one,
                                     one, one, None, None)
        assert (got != invalid) == ok


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq", [1, 4, 48])
def test_attend_of_views_with_one_entry(Hq, dtype):
    """One token's queries out of rows of odd length, and a cache whose only page
    and only head have strides of 3 and 5 (48 heads go to the kernel for many rows)."""
    t = build([(1, 9)], Hq, 1, 64, 16, dtype, seed=Hq)
    pages = t["k"].shape[0]
    t["q"] = t["q"].as_strided((1, Hq, 64), (Hq * 64 + 1, 64, 1))
    at = int(t["table"][0, 0])
    t["k"], t["v"] = (t[c][at:at + 1].as_strided((1, 16, 1, 64), (3, 64, 5, 1),
                                                 t[c][at:at + 1].storage_offset()) for c in "kv")
    assert pages > 1
    t["table"].zero_()
    check(t)


@pytest.mark.gpu
def test_append_and_verify_of_views_with_one_entry():
    from paper_2608_11368_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(0)
    k = torch.zeros((1, 16, 1, 64), device="cuda").as_strided((1, 16, 1, 64), (3, 64, 5, 1))
    v = torch.zeros((1, 16, 1, 64), device="cuda")
    kv = torch.randn((2, 64), generator=g, device="cuda")
    new = [kv[x].as_strided((1, 1, 64), (7, 9, 1), 64 * x) for x in range(2)]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pair_cache_append(*new, torch.tensor([5], device="cuda"), k, v, dev_err=err)
    assert torch.equal(k[0, 5, 0], kv[0]) and torch.equal(v[0, 5, 0], kv[1])
    p = torch.softmax(torch.randn((99, 1), generator=g, device="cuda"), 0)
    i32 = dict(dtype=torch.int32, device="cuda")
    rest = (torch.zeros(1, **i32), torch.tensor([0, 1], **i32), torch.zeros(1, device="cuda"),
            torch.full((1,), 0.4, device="cuda"))
    got = B.pair_verify_drafts(p.t(), *rest, dev_err=err)
    want = B.pair_verify_drafts(p.t().reshape(1, 99).clone(), *rest, dev_err=err)
    assert p.t().stride(0) < 99 and all(torch.equal(x, y) for x, y in zip(got, want))
    assert B.pair_status_sync(err) == 0
