"""pair_cache_append_q8 and pair_cache_read_q8 against the 64-bit form: codes and
exponent bytes are equal, values read back are exact."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu

CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def empty_cache(pages, page, H, D, fmt, layout="token", seed=0):
    """Codes and exponent bytes with random contents, and views by token or head."""
    rng = np.random.default_rng(seed)
    shape = (pages, page, H, D) if layout == "token" else (pages, H, page, D)
    c = torch.from_numpy(rng.integers(0, 256, shape).astype(np.uint8)).cuda().view(CODES[fmt])
    e = torch.from_numpy(rng.integers(0, 256, shape[:3]).astype(np.uint8)).cuda()
    return (c, e) if layout == "token" else (c.permute(0, 2, 1, 3), e.permute(0, 2, 1))


def rows(T, H, D, dtype, seed):
    """New rows of all sizes: ordinary ones, zeros, ones around the largest codes,
    tiny and huge ones, ones with a NaN or an infinity. Returns k, v as views of one
    array, as a projection leaves them."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, 2, H, D)) * np.exp(2 * rng.standard_normal((T, 2, H, 1)))
    kind = rng.integers(0, 12, (T, 2, H))
    x[kind == 0] = 0.0
    x[kind == 1] *= 2.0 ** -126
    x[kind == 2] *= 2.0 ** 118
    for k, edge in ((3, 127.5), (4, 464.0)):  # the border of the exponent, and ties
        at = kind == k
        n = int(at.sum())
        near = edge * (1 + rng.integers(-2, 3, (n, D)) * 2.0 ** -8)
        x[at] = np.where(rng.random((n, D)) < 0.2, near, rng.integers(-900, 900, (n, D)) / 4)
        x[at] *= 2.0 ** rng.integers(-20, 20, (n, 1))
    y = torch.from_numpy(x).to(dtype).cuda()
    odd = rng.integers(0, 30, (T, 2, H))
    for k, value in ((0, float("nan")), (1, float("inf")), (2, -float("inf"))):
        for t, c, h in zip(*np.nonzero(odd == k)):
            y[t, c, h, int(rng.integers(D))] = value
    return y[:, 0], y[:, 1]


def f64(x):
    return x.double().cpu().numpy()


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,D,page,layout", [
    (1, 1, 64, 1, "token"), (5, 3, 16, 7, "token"), (64, 8, 128, 16, "token"),
    (333, 8, 128, 16, "head"), (100, 2, 80, 24, "head"), (70, 5, 256, 16, "token"),
    (40, 1, 240, 64, "head"), (50, 40, 48, 8, "token")])
def test_append_and_read(T, H, D, page, layout, dtype, fmt):
    from paper_2608_11368_gb300 import binding as B
    rng = np.random.default_rng(T)
    pages = -(-T // page) + 3
    kc, ke = empty_cache(pages, page, H, D, fmt, layout, 1)
    vc, ve = empty_cache(pages, page, H, D, fmt, "token", 2)
    before = [x.clone() for x in (kc.view(torch.uint8), ke, vc.view(torch.uint8), ve)]
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    slots[rng.random(T) < 0.1] = -1
    k, v = rows(T, H, D, dtype, T)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ds = torch.from_numpy(slots).cuda()
    B.pair_cache_append_q8(k, v, ds, kc, ke, vc, ve, dev_err=err)
    assert B.pair_last_launch_count() == 1
    there = slots >= 0
    at = (slots[there] // page, slots[there] % page)
    for x, c, e, c0, e0 in ((k, kc, ke, *before[:2]), (v, vc, ve, *before[2:])):
        want_c, want_e = rollout.store_q8(f64(x)[there], fmt)
        got_e = e.cpu().numpy()
        assert np.array_equal(got_e[at], want_e)
        got = c.to(torch.float32).cpu().numpy()
        assert np.array_equal(got[at], want_c)
        mask = np.ones((pages, page), bool)  # everything else as it was
        mask[at] = False
        assert np.array_equal(got_e[mask], e0.cpu().numpy()[mask])
        raw = c.view(torch.uint8).cpu().numpy()
        assert np.array_equal(raw[mask], c0.cpu().numpy()[mask])
    # Back: some slots twice, in another order.
    pick = np.concatenate([rng.permutation(T), rng.integers(0, T, 5)])
    back = slots[pick]
    for out in (torch.float32, torch.bfloat16):
        got = B.pair_cache_read_q8(torch.from_numpy(back).cuda(), kc, ke, vc, ve, dtype=out,
                                   dev_err=err)
        for x, g in zip((k, v), got):
            want = rollout.values_q8(*rollout.store_q8(f64(x)[pick], fmt))
            want[back < 0] = 0.0
            want = torch.from_numpy(want).to(out).double().numpy()  # exact but for tiny ones
            assert g.shape == (T + 5, H, D) and g.dtype is out
            assert np.array_equal(f64(g), want, equal_nan=True)
    assert B.pair_status_sync(err) == 0


@pytest.mark.parametrize("fmt", sorted(CODES))
def test_every_code_reads_back(fmt):
    """All bytes but e4m3's two NaN ones, under every exponent byte."""
    from paper_2608_11368_gb300 import binding as B
    raw = torch.arange(256, dtype=torch.int32, device="cuda").to(torch.uint8)
    codes = raw.view(1, 1, 1, 256).expand(256, 1, 1, 256).contiguous().view(CODES[fmt])
    exps = raw.view(256, 1, 1).contiguous()
    c64 = f64(codes.to(torch.float32))[:, :, 0]
    fine = np.isfinite(c64[0, 0])
    assert fine.sum() == (256 if fmt == "i8" else 254)
    want = rollout.values_q8(c64, np.arange(256)[:, None])
    for out in (torch.float32, torch.bfloat16):
        k, v = B.pair_cache_read_q8(torch.arange(256, device="cuda"), codes, exps, codes, exps,
                                    dtype=out)
        w = torch.from_numpy(want).to(out).double().numpy()
        for g in (k, v):
            assert np.array_equal(f64(g)[..., fine], w[..., fine], equal_nan=True)


@pytest.mark.parametrize("fmt", sorted(CODES))
def test_slots_that_do_not_exist(fmt):
    """Reported, left out, and read as zeros."""
    from paper_2608_11368_gb300 import binding as B
    pages, page, H, D = 3, 4, 2, 64
    kc, ke = empty_cache(pages, page, H, D, fmt)
    vc, ve = empty_cache(pages, page, H, D, fmt, seed=1)
    before = [x.clone() for x in (kc.view(torch.uint8), ke, vc.view(torch.uint8), ve)]
    k, v = rows(4, H, D, torch.float32, 0)
    slots = torch.tensor([-2, pages * page, 2 ** 40, -1], device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pair_cache_append_q8(k, v, slots, kc, ke, vc, ve, dev_err=err)
    assert B.pair_status_sync(err) == 10
    for x, y in zip((kc.view(torch.uint8), ke, vc.view(torch.uint8), ve), before):
        assert torch.equal(x, y)
    gk, gv = B.pair_cache_read_q8(slots, kc, ke, vc, ve, dev_err=err)
    assert B.pair_status_sync(err) == 10
    assert not gk.any() and not gv.any()
    B.pair_cache_read_q8(slots[3:], kc, ke, vc, ve, dev_err=err)
    assert B.pair_status_sync(err) == 0


def test_read_into_views_and_refusals():
    """Outputs that are rows of a wider array; what the binding refuses."""
    from paper_2608_11368_gb300 import binding as B
    kc, ke = empty_cache(4, 8, 2, 64, "i8")
    vc, ve = empty_cache(4, 8, 2, 64, "i8", seed=3)
    ke.fill_(120), ve.fill_(121)
    slots = torch.tensor([3, -1, 17], device="cuda")
    wide = torch.full((3, 2, 2, 72), 7.0, device="cuda")
    B.pair_cache_read_q8(slots, kc, ke, vc, ve, k=wide[:, 0, :, :64], v=wide[:, 1, :, :64])
    k, v = B.pair_cache_read_q8(slots, kc, ke, vc, ve, dtype=torch.float32)
    assert torch.equal(wide[:, 0, :, :64], k) and torch.equal(wide[:, 1, :, :64], v)
    assert (wide[..., 64:] == 7).all()
    for args in ((slots.int(), kc, ke, vc, ve), (slots, kc.float(), ke, vc, ve),
                 (slots, kc, ke.int(), vc, ve), (slots, kc, ke, vc.view(torch.float8_e4m3fn), ve),
                 (slots, kc, ke[:3], vc, ve), (slots, kc, ke, vc[:, :7], ve),
                 (slots, kc, ke.cpu(), vc, ve)):
        with pytest.raises((TypeError, ValueError)):
            B.pair_cache_read_q8(*args)
    with pytest.raises(TypeError):
        B.pair_cache_read_q8(slots, kc, ke, vc, ve, dtype=torch.float16)
    with pytest.raises(ValueError):
        B.pair_cache_append_q8(k, v, slots, kc[..., :48], ke, vc[..., :48], ve)


def test_append_on_another_stream_and_captured():
    """A captured append and read, replayed with other rows and slots."""
    from paper_2608_11368_gb300 import binding as B
    kc, ke = empty_cache(8, 16, 2, 128, "e4m3")
    vc, ve = empty_cache(8, 16, 2, 128, "e4m3", seed=1)
    T = 37
    k, v = (x.contiguous() for x in rows(T, 2, 128, torch.bfloat16, 0))
    slots = torch.arange(T, device="cuda")
    out = [torch.zeros((T, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def step():
        B.pair_cache_append_q8(k, v, slots, kc, ke, vc, ve)
        B.pair_cache_read_q8(slots, kc, ke, vc, ve, k=out[0], v=out[1])

    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    k2, v2 = rows(T, 2, 128, torch.bfloat16, 9)
    k.copy_(k2), v.copy_(v2), slots.copy_(torch.randperm(128, device="cuda")[:T])
    graph.replay()
    torch.cuda.synchronize()
    for x, g in zip((k2, v2), out):
        want = rollout.values_q8(*rollout.store_q8(f64(x), "e4m3"))
        want = torch.from_numpy(want).bfloat16().double().numpy()
        assert np.array_equal(f64(g), want, equal_nan=True)
