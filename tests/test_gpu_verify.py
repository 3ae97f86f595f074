"""pair_verify_drafts: emitted tokens equal to the definition's everywhere,
log-probabilities within logf's 2 ulp plus one rounding; and, over many draws,
tokens distributed as the target's."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def case(K, V, dtype, with_q, seed, spare=0, pad=0):
    """Requests with K[i] drafts (-1: an empty chunk)."""
    rng = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(np.asarray(K) + 1)]).astype(np.int32)
    T = max(1, int(cu[-1]) + spare)
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = 3.0 * torch.randn((T, V), generator=g, device="cuda")
    p = torch.full((T, V + pad), float("nan"), dtype=dtype, device="cuda")
    p[:, :V] = torch.softmax(z, -1)
    d = torch.softmax(z + 0.7 * torch.randn((T, V), generator=g, device="cuda"), -1)
    q = torch.full((T, V + pad), float("nan"), dtype=dtype, device="cuda")
    q[:, :V] = d
    ids = torch.multinomial(d if with_q else torch.softmax(2 * z, -1), 1,
                            generator=g)[:, 0].to(torch.int32).roll(1)
    return dict(p=p[:, :V], q=q[:, :V] if with_q else None, ids=ids, cu=dev(cu),
                u=dev(rng.random(T, dtype=np.float32)),
                ud=dev(rng.random(len(K), dtype=np.float32)))


def check(c):
    from paper_2608_11368_gb300 import binding as B
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids, logp, n = B.pair_verify_drafts(c["p"], c["ids"], c["cu"], c["u"], c["ud"], q=c["q"],
                                        dev_err=err)
    word = int(err)
    err.zero_()
    f = lambda x: None if x is None else x.float().cpu().numpy()  # noqa: E731
    want = rollout.verify_drafts(f(c["p"]), c["ids"].cpu().numpy(), c["cu"].cpu().numpy(),
                                 f(c["u"]), f(c["ud"]), f(c["q"]))
    assert np.array_equal(ids.cpu().numpy(), want["ids"])
    assert np.array_equal(n.cpu().numpy(), want["n"])
    lp = logp.double().cpu().numpy()
    assert (np.abs(lp - want["logp"]) <= 3 * 2.0 ** -23 * np.abs(want["logp"]) + 2.0 ** -149).all()
    assert (word & 2 != 0) == want["bad_id"] and (word & 64 != 0) == want["bad_p"]
    return want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("K,V,pad", [
    ([0], 1, 0), ([1], 2, 0), ([4], 1000, 0), ([4, 4, 4, 4], 4099, 0), ([0, 3, -1, 7, 1], 513, 3),
    ([40], 130, 1), ([33, -1, 65], 257, 7), ([2] * 200, 997, 0), ([1] * 1300, 64, 5)])
def test_verify(K, V, pad, with_q, dtype):
    want = check(case(K, V, dtype, with_q, seed=len(K) + V, spare=len(K) % 3, pad=pad))
    if len(K) > 100:  # every way of ending occurs
        assert 0 < (want["n"] == 1).sum() < len(K) and (want["n"] == np.asarray(K) + 1).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verify_rows_that_lie_differently(dtype):
    """q's rows begin at another place within 16 bytes than p's."""
    c = case([3, 0, 5, -1, 2], 1001, dtype, True, seed=6)
    wide = torch.full((c["q"].shape[0], 1010), float("nan"), dtype=dtype, device="cuda")
    wide[:, 3:1004] = c["q"]
    check(dict(c, q=wide[:, 3:1004]))
    check(dict(c, p=wide[:, 3:1004], q=c["p"].contiguous()))


@pytest.mark.parametrize("y", [0, 1, 3, 4, 7, 8, 511, 512, 998, 999])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verify_looked_up_draft_anywhere_in_the_row(y, dtype):
    c = case([1] * 40, 1000, dtype, False, seed=y)
    c["ids"][:] = y
    c["u"][:] = 1.0  # never accepted: drawn from p without the draft
    want = check(c)
    assert (want["n"] == 1).all() and not (want["ids"] == y).any()


@pytest.mark.parametrize("with_q", [True, False])
def test_verify_large_vocabulary(with_q):
    check(case([3, 3], 151936, torch.float32, with_q, seed=4))


def test_verify_ends_of_the_draw():
    """u_draw at 0 and just below 1, weights that end in zeros, one weight."""
    V = 300
    p = np.zeros((6, V), np.float32)
    p[:, 7], p[:, 250] = 0.25, 0.75
    p[4] = 0
    p[4, 299] = 1
    p[5] = 0
    p[5, 0] = 1
    top = np.nextafter(np.float32(1), np.float32(0))
    c = dict(p=dev(p), q=None, ids=dev(np.zeros(6, np.int32)), cu=dev(np.arange(7, dtype=np.int32)),
             u=dev(np.zeros(6, np.float32)),
             ud=dev(np.array([0, top, 0.25, np.nextafter(np.float32(0.25), np.float32(0)), top, top],
                             np.float32)))
    want = check(c)
    assert want["ids"].tolist() == [7, 250, 250, 7, 299, 0]


def test_verify_equal_distributions_and_nothing_left():
    """p = q: a draft that the rounding of u q still refuses leaves no
    difference, and p alone is drawn from; a row of zeros is reported."""
    V = 1000
    rng = np.random.default_rng(0)
    x = rng.random((4, V)).astype(np.float32)
    x /= x.sum(1, keepdims=True)
    c = dict(p=dev(x), q=dev(x), ids=dev(np.array([5, 6, 7, 8], np.int32)),
             cu=dev(np.array([0, 2, 4], np.int32)), u=dev(np.array([1.0, 0, 0.5, 0], np.float32)),
             ud=dev(np.array([0.3, 0.9], np.float32)))
    check(c)
    zero = dict(c, p=dev(np.zeros((4, V), np.float32)), q=None)
    assert check(zero)["bad_p"]
    nan = x.copy()
    nan[0] = np.nan
    nan[2, ::2] = np.nan
    want = check(dict(c, p=dev(nan), u=dev(np.ones(4, np.float32))))
    assert want["bad_p"] and want["n"].tolist() == [0, 1]


def test_verify_drafts_out_of_range():
    c = case([3, 2], 500, torch.float32, True, seed=1)
    for bad in (-1, 500, 2 ** 31 - 1, -2 ** 31):
        for with_q in (True, False):
            x = dict(c, ids=c["ids"].clone(), q=c["q"] if with_q else None)
            x["ids"][1] = bad
            assert check(x)["bad_id"]


def test_verify_offsets_that_do_not_fit():
    from paper_2608_11368_gb300 import binding as B
    c = case([1, 1], 100, torch.float32, True, seed=1)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for cu in ([0, 2, 1], [0, 2, 5], [0, -1, 4]):
        B.pair_verify_drafts(c["p"], c["ids"], dev(np.array(cu, np.int32)), c["u"], c["ud"],
                             q=c["q"], dev_err=err)
        assert B.STATUS_NAMES[B.pair_status_sync(err)] == "PAIR_ERR_PAGES"


def test_verify_emits_the_target_distribution():
    """First emitted token over 40,000 requests with the same p and q: counts
    within 5 sigma of the target's probabilities (chance of a failure for a
    right kernel: 12 categories x 6e-7)."""
    from paper_2608_11368_gb300 import binding as B
    N, V = 40000, 12
    rng = np.random.default_rng(7)
    p1, q1 = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    p = dev(np.tile(p1.astype(np.float32), (2 * N, 1)))
    q = dev(np.tile(q1.astype(np.float32), (2 * N, 1)))
    ids = np.zeros(2 * N, np.int32)
    ids[1::2] = rng.choice(V, N, p=q1)
    cu = dev((2 * np.arange(N + 1)).astype(np.int32))
    out, _, n = B.pair_verify_drafts(p, dev(ids), cu, dev(rng.random(2 * N, dtype=np.float32)),
                                     dev(rng.random(N, dtype=np.float32)), q=q)
    first = np.bincount(out.cpu().numpy()[::2], minlength=V)
    sigma = np.sqrt(N * p1 * (1 - p1))
    assert (np.abs(first - N * p1) <= 5 * sigma + 1).all()
    accepted = (n.cpu().numpy() == 2).mean()
    overlap = np.minimum(p1, q1).sum()
    assert abs(accepted - overlap) <= 5 * np.sqrt(overlap * (1 - overlap) / N)


def test_verify_refuses():
    from paper_2608_11368_gb300 import binding as B
    c = case([1, 1], 100, torch.float32, True, seed=1)

    def refuses(kind, **change):
        x = dict(c, **change)
        with pytest.raises(kind):
            B.pair_verify_drafts(x["p"], x["ids"], x["cu"], x["u"], x["ud"], q=x["q"])

    refuses(TypeError, p=c["p"].double())
    refuses(TypeError, q=c["q"].bfloat16())
    refuses(ValueError, q=c["q"][:, :99])
    refuses(TypeError, ids=c["ids"].long())
    refuses(ValueError, ids=c["ids"][:3])
    refuses(ValueError, ud=c["ud"][:1])
    refuses(ValueError, p=c["p"].t().contiguous().t())
