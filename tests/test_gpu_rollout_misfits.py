"""Requests and rows that do not fit, or that nobody owns: what the others get."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.parametrize("count", [0, 1, 2, 3])
def test_extend_serves_who_needs_no_page_after_pages_ran_out(count):
    """By hand: requests 0 and 2 want one and three pages, 1 and 3 have room in
    the pages that they hold."""
    from paper_2608_11368_gb300 import binding as B
    err, tab = i32([0]), i32([[0, -1, -1, -1], [1, -1, -1, -1], [2, -1, -1, -1], [3, 4, -1, -1]])
    kv, held, cu, slots, taken = B.pair_pages_extend(
        i32([16, 3, 16, 20]), i32([1, 1, 1, 2]), i32([1, 5, 40, 3]), i32([7, 8, 9]), i32([count]),
        tab, 16, 60, dev_err=err)
    assert B.STATUS_NAMES[B.pair_status_sync(err)] == "PAIR_ERR_PAGES"
    first = count > 0
    assert kv.tolist() == [17 if first else 16, 8, 16, 23]
    assert held.tolist() == [2 if first else 1, 1, 1, 2]
    assert cu.tolist() == [0, 1, 6, 46, 49]
    assert slots.tolist() == ([7 * 16 if first else -1] + [16 + x for x in range(3, 8)] + [-1] * 40
                              + [4 * 16 + x for x in (4, 5, 6)] + [-1] * 11)
    assert taken.tolist() == [int(first)]
    assert tab.tolist() == [[0, 7 if first else -1, -1, -1], [1, -1, -1, -1], [2, -1, -1, -1],
                            [3, 4, -1, -1]]


def test_extend_pages_go_in_the_requests_order():
    """By hand: behind a request whose pages run out, no other one is given any."""
    from paper_2608_11368_gb300 import binding as B
    err, tab = i32([0]), i32([[0, -1, -1], [1, -1, -1], [2, -1, -1]])
    kv, held, cu, slots, taken = B.pair_pages_extend(
        i32([16, 16, 16]), i32([1, 1, 1]), i32([1, 32, 1]), i32([7, 8]), i32([2]), tab, 16, 40,
        dev_err=err)
    assert B.STATUS_NAMES[B.pair_status_sync(err)] == "PAIR_ERR_PAGES"
    assert kv.tolist() == [17, 16, 16] and held.tolist() == [2, 1, 1] and taken.tolist() == [1]
    assert slots.tolist() == [7 * 16] + [-1] * 39


def test_extend_many_requests_after_pages_ran_out():
    """As above over several blocks of tokens and runs of requests: the pages end
    at some request; the ones that need none are served wherever they are."""
    from paper_2608_11368_gb300 import binding as B
    R, page, n = 3000, 16, 3
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 40, R)
    held = -(-lens // page)
    need = np.maximum(-(-(lens + n) // page) - held, 0)
    table = np.full((R, 4), -1)
    table[np.arange(4) < held[:, None]] = np.arange(held.sum())
    free = np.arange(held.sum(), held.sum() + need.sum())
    count = int(need.sum()) // 3
    before = np.cumsum(need) - need
    ok = (need == 0) | (before + need <= count)
    assert (~ok).any() and ok[np.argmin(ok):].any()
    err, tab = i32([0]), i32(table)
    kv, ho, cu, slots, taken = B.pair_pages_extend(
        i32(lens), i32(held), i32([n] * R), i32(free), i32([count]), tab, page, R * n, dev_err=err)
    assert B.STATUS_NAMES[B.pair_status_sync(err)] == "PAIR_ERR_PAGES"
    assert np.array_equal(kv.cpu(), np.where(ok, lens + n, lens))
    assert np.array_equal(ho.cpu(), held + np.where(ok, need, 0))
    for i in range(R):
        if ok[i]:
            table[i, held[i]:held[i] + need[i]] = free[before[i]:before[i] + need[i]]
    assert np.array_equal(tab.cpu(), table) and int(taken) == (before + need)[ok & (need > 0)].max()
    pos = lens[:, None] + np.arange(n)
    want = np.take_along_axis(table, np.minimum(pos // page, 3), 1) * page + pos % page
    assert np.array_equal(slots.cpu(), np.where(ok[:, None], want, -1).ravel())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first", [1, 5, 700])
def test_verify_rows_before_the_first_request(first, dtype):
    """Offsets that begin behind row 0 (some requests of a larger step): the rows
    before belong to nobody and say so, the requests are served."""
    from paper_2608_11368_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(first)
    R, n, V = 6, 3, 500
    T = first + R * n + 2
    p = torch.softmax(3 * torch.randn((T, V), generator=g, device="cuda"), -1).to(dtype)
    q = torch.softmax(3 * torch.randn((T, V), generator=g, device="cuda"), -1).to(dtype)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32)
    u, ud = torch.rand(T, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")
    cu = i32(first + n * np.arange(R + 1))
    err = i32([0])
    out, logp = i32([77] * T), torch.full((T,), 77.0, device="cuda")
    B.pair_verify_drafts(p, ids, cu, u, ud, q=q, out_ids=out, logp=logp, dev_err=err)
    assert B.pair_status_sync(err) == 0
    want = B.pair_verify_drafts(p[first:], ids[first:].contiguous(), cu - first,
                                u[first:].contiguous(), ud, q=q[first:])
    assert (out[:first] == -1).all() and (logp[:first] == 0).all()
    assert torch.equal(out[first:], want[0]) and torch.equal(logp[first:], want[1])
