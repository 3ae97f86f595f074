"""pair_verify_drafts: the exchange between the CTAs of a cluster, from the first
request of a launch on."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("C", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("R", [1, 3])
def test_verify_first_exchange(C, R):
    """Rows as short as a cluster of C CTAs is used for (2048 values each) and
    requests without drafts: the CTAs exchange their sums as soon after their
    start as they ever do. A sum that is lost or late gives another token: each
    CTA holds a like part of the weight, and the draws fall all over the row.
    Many launches, one after the other without a pause."""
    from paper_2608_11368_gb300 import binding as B
    V, N = 2048 * C, 200
    rng = np.random.default_rng(C)
    p = rng.random((R, V), dtype=np.float32)
    p /= p.sum(1, keepdims=True)
    ids, cu, u = np.zeros(R, np.int32), np.arange(R + 1, dtype=np.int32), np.zeros(R, np.float32)
    draws = [rng.random(R, dtype=np.float32) for _ in range(8)]

    def dev(x):
        return torch.from_numpy(x).cuda()

    want = [rollout.verify_drafts(p, ids, cu, u, x) for x in draws]
    args, uds = (dev(p), dev(ids), dev(cu), dev(u)), [dev(x) for x in draws]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = [B.pair_verify_drafts(*args, uds[k % 8], dev_err=err) for k in range(N)]
    assert B.pair_status_sync(err) == 0
    for k, (tok, _, n) in enumerate(got):
        assert np.array_equal(tok.cpu().numpy(), want[k % 8]["ids"])
        assert (n == 1).all()
