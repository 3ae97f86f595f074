"""pair_attend_paged, many rows: tiles whose rows in use end inside a warp, and in
them values that are not finite, so that a warp's lanes part where its rows do."""
import numpy as np
import pytest
import torch

from oracle import rollout
from tests.test_gpu_attend import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (3, 1), (4, 2)])
@pytest.mark.parametrize("reqs", [
    [(33, 33)], [(34, 100), (63, 500), (95, 95)], [(129, 300)], [(161, 161), (200, 1000)],
    [(257, 400), (33, 90)], [(287, 290)], [(65, 9000)], [(100, 20)]])
def test_attend_rows_end_inside_a_warp(reqs, heads, D):
    """Values of later tokens that are not finite (+inf, -inf, NaN, each in a column of
    its own): rows that do not see them are as without, the others take them as
    their sums do. Bound as in test_gpu_attend: weights and output rounded to bf16,
    fp32 sums."""
    from paper_2608_11368_gb300 import binding as B
    Hq, Hkv = heads
    t = build(reqs, Hq, Hkv, D, 16, torch.bfloat16, seed=len(reqs) + D)
    bad = {1: np.inf, 2: -np.inf, 3: np.nan}
    for i, (n, kv) in enumerate(reqs):
        for c, x in bad.items():
            pos = max(0, kv - c * max(1, min(n, kv) // 4))  # the chunk's last quarters begin there
            t["v"][int(t["table"][i, pos // 16]), pos % 16, Hkv - 1, c] = x
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = B.pair_attend_paged(t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"],
                                   dev_err=err)
    assert B.pair_status_sync(err) == 0
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    ro, rl, mag, size = rollout.attend_paged(f(t["q"]), f(t["k"]), f(t["v"]),
                                             t["table"].cpu().numpy(), t["kv"].cpu().numpy(),
                                             t["cu"].cpu().numpy(), D ** -0.5)
    out, lse = f(out), f(lse)
    assert np.isnan(ro).any() or all(n > kv for n, kv in reqs)
    assert np.array_equal(np.isnan(out), np.isnan(ro))
    assert np.array_equal(np.isposinf(out), np.isposinf(ro))
    assert np.array_equal(np.isneginf(out), np.isneginf(ro))
    fin = np.isfinite(ro)
    sums = 2.0 * 2.0 ** -24 * (D * size + int(t["kv"].max()) + 16)
    rel = np.broadcast_to((2 * sums + 2 * 2.0 ** -8 * 1.01)[..., None], ro.shape)
    assert (np.abs(out[fin] - ro[fin]) <= rel[fin] * mag[fin] + 1e-30).all()
    seen = np.isfinite(rl)
    assert np.array_equal(np.isneginf(lse), ~seen)
    assert (np.abs(lse[seen] - rl[seen]) <= sums[seen] + 2.0 ** -22 * np.abs(rl[seen])).all()
