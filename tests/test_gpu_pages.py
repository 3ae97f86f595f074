"""pair_pages_extend and pair_cache_append: whole numbers and copies, equal to
the plain forms everywhere."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def extend(lens, held, n, free, count, table, page, T):
    from paper_2608_11368_gb300 import binding as B
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    tab = i32(table)
    kv, ho, cu, slots, taken = B.pair_pages_extend(i32(lens), i32(held), i32(n), i32(free),
                                                   i32([count]), tab, page, T, dev_err=err)
    st = B.pair_status_sync(err)
    want = rollout.pages_extend(lens, held, n, free, count, np.asarray(table, np.int32), page, T)
    assert (st != 0) == want["error"] and B.STATUS_NAMES[st] in ("PAIR_OK", "PAIR_ERR_PAGES")
    for got, key in ((tab, "table"), (kv, "kv_len"), (ho, "held"), (cu, "cu"), (slots, "slots")):
        assert np.array_equal(got.cpu().numpy().astype(np.int64), want[key].astype(np.int64)), key
    assert int(taken) == want["taken"]
    return want


def random_case(rng, R, page, len_hi, n_hi, extra=0.2):
    lens, n = rng.integers(0, len_hi + 1, R), rng.integers(0, n_hi + 1, R)
    held = -(-lens // page) + (rng.random(R) < extra)
    need = np.maximum(-(-(lens + n) // page) - held, 0)
    width = int((held + need).max()) + 1
    total = int((held + need).sum()) + 5
    order = rng.permutation(total)
    table = np.full((R, width), -1)
    at = 0
    for i in range(R):
        table[i, :held[i]] = order[at:at + held[i]]
        at += int(held[i])
    return lens, held, n, order[at:], total - at, table, int(n.sum())


@pytest.mark.parametrize("R,page,len_hi,n_hi", [
    (1, 16, 0, 1), (1, 16, 700, 1), (1, 8, 5, 5000), (7, 1, 30, 9), (64, 16, 2048, 1),
    (33, 24, 100, 40), (1025, 16, 300, 3), (1024, 64, 40, 300), (5000, 16, 50, 2), (300, 128, 0, 7)])
def test_extend(R, page, len_hi, n_hi):
    rng = np.random.default_rng(R + page)
    lens, held, n, free, count, table, total = random_case(rng, R, page, len_hi, n_hi)
    want = extend(lens, held, n, free, count, table, page, max(1, total) + R % 3)
    assert not want["error"]


def test_extend_stopped_requests_take_nothing():
    want = extend([16, 17, 5], [1, 2, 1], [0, 0, 0], [9], 1, [[0, -1], [1, 2], [3, -1]], 16, 4)
    assert want["taken"] == 0 and (want["slots"] == -1).all()


@pytest.mark.parametrize("count", [0, 1, 2, 3, -4, 100])
def test_extend_pages_run_out(count):
    # A count beyond the list is cut to it; later requests that need none go on.
    extend([16, 3, 16, 20], [1, 1, 1, 2], [1, 5, 40, 3], [7, 8, 9], count,
           [[0, -1, -1, -1], [1, -1, -1, -1], [2, -1, -1, -1], [3, 4, -1, -1]], 16, 60)


@pytest.mark.parametrize("lens,held,n", [
    ([-1, 4], [1, 1], [1, 1]), ([4, 4], [-1, 1], [1, 1]), ([4, 4], [1, 1], [-3, 1]),
    ([40, 4], [1, 1], [1, 1]), ([4, 4], [5, 1], [1, 1]), ([4, 4], [1, 1], [100, 1]),
    ([2 ** 31 - 1, 4], [2, 1], [1, 1])])
def test_extend_entries_that_do_not_fit(lens, held, n):
    extend(lens, held, n, [7, 8, 9], 3, [[0, 1], [2, 3]], 16, 110)


def test_extend_rows_that_do_not_fit():
    extend([4, 4, 4], [1, 1, 1], [3, 3, 0], [7, 8, 9], 3, [[0, 1], [2, 3], [4, 5]], 16, 4)


def test_extend_slots_beyond_32_bits():
    page = 2 ** 20
    want = extend([5], [1], [3], [1], 1, [[2 ** 31 - 2]], page, 3)
    assert want["slots"][0] == (2 ** 31 - 2) * page + 5


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("T,H,D,page", [(1, 1, 64, 16), (5, 3, 128, 24), (700, 8, 128, 16),
                                        (64, 2, 8, 1), (33, 5, 256, 7)])
def test_append(T, H, D, page, layout, dtype):
    from paper_2608_11368_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(T)
    pages = -(-T // page) + 3
    shape = (pages, page, H, D) if layout == "token" else (pages, H, page, D)
    k, v = (torch.randn(shape, generator=g, device="cuda").to(dtype) for _ in range(2))
    if layout == "head":
        k, v = k.permute(0, 2, 1, 3), v.permute(0, 2, 1, 3)
    kv = torch.randn((T, 2, H, D), generator=g, device="cuda").to(dtype)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:T]
    slots[torch.rand(T, generator=g, device="cuda") < 0.2] = -1
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    wk, wv = k.clone(), v.clone()
    for t, s in enumerate(slots.tolist()):
        if s >= 0:
            wk[s // page, s % page], wv[s // page, s % page] = kv[t, 0], kv[t, 1]
    ok, ov = B.pair_cache_append(kv[:, 0], kv[:, 1], slots, k, v, dev_err=err)
    assert B.pair_status_sync(err) == 0
    assert torch.equal(ok, wk) and torch.equal(ov, wv) and ok.data_ptr() == k.data_ptr()
    # Slots outside the cache are reported and left out.
    for bad in (-2, pages * page, 2 ** 62, -2 ** 63):
        s2 = torch.full_like(slots, -1)
        s2[0] = bad
        B.pair_cache_append(kv[:, 0], kv[:, 1], s2, k, v, dev_err=err)
        assert B.STATUS_NAMES[B.pair_status_sync(err)] == "PAIR_ERR_PAGES"
        assert torch.equal(k, wk) and torch.equal(v, wv)


def test_pages_and_append_refuse():
    from paper_2608_11368_gb300 import binding as B
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    c = torch.zeros((3, 16, 2, 64), dtype=torch.bfloat16, device="cuda")
    s = torch.zeros(4, dtype=torch.int64, device="cuda")
    with pytest.raises(TypeError):
        B.pair_cache_append(x, x.float(), s, c, c)
    with pytest.raises(TypeError):
        B.pair_cache_append(x, x, s.int(), c, c)
    with pytest.raises(ValueError):
        B.pair_cache_append(x, x, s, c[:, :, :1], c[:, :, :1])
    with pytest.raises(ValueError):
        B.pair_cache_append(x.transpose(1, 2), x.transpose(1, 2), s, c, c)
    with pytest.raises(B.PairError):
        B.pair_cache_append(x[:, :, 4:], x[:, :, 4:], s, c[..., 4:], c[..., 4:])  # 8-byte aligned
    one, tab = i32([1]), i32([[0, 1]])
    with pytest.raises(TypeError):
        B.pair_pages_extend(one.long(), one, one, one, one, tab, 16, 1)
    with pytest.raises(ValueError):
        B.pair_pages_extend(one, i32([1, 1]), one, one, one, tab, 16, 1)
    for page, T in ((0, 1), (16, 0)):
        with pytest.raises((B.PairError, ValueError)):
            B.pair_pages_extend(one, one, one, one, one, tab, page, T)
