"""pair_attend_paged_q8 against the 64-bit form over the stored values: single
tokens, drafted chunks and long chunks, head layouts, page sizes, cache orders, rows
that see nothing, whatever lies in places that are not seen.

The stored values are exact in every arithmetic that the kernels use (whole numbers
or e4m3 times a power of two), so the error bounds are those of attention over a bf16
or fp32 cache, from the same steps. fp32: a score is a dot product of D terms, off by
at most D 2^-24 size (size = scale sum |q_d k_d|); sums over m keys add m 2^-24,
exponentials and rescalings 16 2^-24; relative to mag = sum p |v| twice (weights and
normaliser). bf16: scores with twice the unit (accumulation on the tensor cores need
not round to nearest), weights and output rounded once each, by up to eps / 2 = 2^-8
relative to mag and to |out| <= mag."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu

CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}


def build(reqs, Hq, Hkv, D, page, dtype, fmt, layout="token", seed=0, spare=0, shared=0, odd=True):
    """Device inputs for requests [(n, kv)]; pages in random order. What nobody
    owns holds random codes under NaN exponents."""
    rng = np.random.default_rng(seed)
    R = len(reqs)
    need = [-(-kv // page) for _, kv in reqs]
    own = [max(x - shared, 0) for x in need]
    pages = sum(own) + shared + 2
    order = rng.permutation(pages)
    table = np.zeros((R, max(1, max(need))), np.int32)
    at = shared
    for i in range(R):
        table[i, :min(shared, need[i])] = order[:min(shared, need[i])]
        table[i, shared:need[i]] = order[at:at + own[i]]
        at += own[i]
    cu = np.concatenate([[0], np.cumsum([n for n, _ in reqs])])
    T = max(1, int(cu[-1]) + spare)
    used = np.zeros((pages, page), bool)
    for i, (_, kv) in enumerate(reqs):
        pos = np.arange(kv)
        used[table[i][pos // page], pos % page] = True
    held = []
    for _ in "kv":
        x = rng.standard_normal((pages, page, Hkv, D))
        x *= np.exp(0.5 * rng.standard_normal((pages, page, Hkv, 1)))
        c, e = rollout.store_q8(x, fmt)
        if fmt == "i8":
            raw = c.astype(np.int8).view(np.uint8)
        else:
            raw = torch.from_numpy(c).to(torch.float8_e4m3fn).view(torch.uint8).numpy().copy()
        raw[~used] = rng.integers(0, 256, raw[~used].shape) if odd else 0
        e[~used] = 255 if odd else 0
        e = e.astype(np.uint8)
        if layout == "head":
            c = torch.from_numpy(np.ascontiguousarray(raw.transpose(0, 2, 1, 3))).cuda()
            e = torch.from_numpy(np.ascontiguousarray(e.transpose(0, 2, 1))).cuda()
            held += [c.view(CODES[fmt]).permute(0, 2, 1, 3), e.permute(0, 2, 1)]
        else:
            held += [torch.from_numpy(raw).cuda().view(CODES[fmt]), torch.from_numpy(e).cuda()]
    q = torch.from_numpy(2.0 * rng.standard_normal((T, Hq, D))).cuda().to(dtype)
    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    return dict(q=q, held=held, table=i32(table), kv=i32([kv for _, kv in reqs]), cu=i32(cu))


def reference(t, scale):
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    k, ke, v, ve = t["held"]
    # NaN codes lie in places that nobody owns only; a NaN exponent says so anyway.
    vals = [rollout.values_q8(np.nan_to_num(f(c.to(torch.float32))), e.cpu().numpy())
            for c, e in ((k, ke), (v, ve))]
    return rollout.attend_paged(f(t["q"]), *vals, t["table"].cpu().numpy(), t["kv"].cpu().numpy(),
                                t["cu"].cpu().numpy(), scale)


def check(t, scale=None, rows=None, ref=None, lost=0.0, **kw):
    from paper_2608_11368_gb300 import binding as B
    D = t["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = B.pair_attend_paged_q8(t["q"], *t["held"], t["table"], t["kv"], t["cu"],
                                      scale=scale, dev_err=err, **kw)
    assert B.pair_status_sync(err) == 0
    ro, rl, mag, size = reference(t, scale) if ref is None else ref
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    m = int(t["kv"].max())
    bf = t["q"].dtype == torch.bfloat16
    sums = (2.0 if bf else 1.0) * 2.0 ** -24 * (D * size + m + 16)
    rel = 2 * sums + (2 * 2.0 ** -8 * 1.01 if bf else 0.0)
    if rows is None:
        rows = np.ones(len(out), bool)
    assert not np.isnan(out[rows]).any()
    assert (np.isinf(lse) == np.isinf(rl))[rows].all()
    fin = np.isfinite(rl) & rows[:, None]
    assert (out[~np.isfinite(rl) & rows[:, None]] == 0).all()
    lse_all, lse, rl = lse, np.where(fin, lse, 0.0), np.where(fin, rl, 0.0)
    assert (np.abs(lse - rl)[fin] <= sums[fin] + 2.0 ** -22 * np.abs(rl[fin])).all()
    assert (np.abs(out - ro)[fin] <= (rel[..., None] * mag)[fin] + 1e-30 + lost).all()
    return out, lse_all


SHAPES = {
    "token": [(1, 1)],
    "tokens": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65), (1, 700)],
    "drafts": [(5, 5), (5, 64), (3, 130), (8, 8), (2, 1000), (5, 257)],
    "chunk": [(40, 40), (129, 300), (1, 77), (64, 64)],
    "long": [(300, 700), (257, 257)],
    "none": [(0, 0), (0, 33), (4, 2), (1, 0), (3, 3), (0, 5), (130, 7)],
}


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (3, 3, 128), (10, 2, 64), (2, 1, 256)])
@pytest.mark.parametrize("what", sorted(SHAPES))
def test_attend(what, heads, dtype, fmt):
    Hq, Hkv, D = heads
    check(build(SHAPES[what], Hq, Hkv, D, 16, dtype, fmt, seed=len(what)))


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("heads", [(8, 4, 64), (8, 8, 128), (16, 4, 128), (32, 8, 64), (8, 4, 256)])
@pytest.mark.parametrize("what", ["tokens", "drafts", "chunk", "none"])
def test_attend_key_heads_in_fours(what, heads, fmt):
    """Four key heads are worked on side by side."""
    Hq, Hkv, D = heads
    check(build(SHAPES[what], Hq, Hkv, D, 16, torch.bfloat16, fmt, seed=len(what)))


@pytest.mark.parametrize("rows", [1, 8, 9, 16, 17, 24, 25, 32, 33])
@pytest.mark.parametrize("hint", [True, False])
def test_attend_every_number_of_rows(rows, hint):
    """Rows of a key head from 1 to more than the kernels for few rows take, known to
    the host or not."""
    check(build([(rows, 200 + rows), (rows, rows), (0, 9), (rows, 70 + rows)], 4, 4, 128, 16,
                torch.bfloat16, "i8", seed=rows), max_new=rows if hint else 0)


@pytest.mark.parametrize("page", [1, 5, 8, 24, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype,fmt", [(torch.bfloat16, "i8"), (torch.bfloat16, "e4m3"),
                                       (torch.float32, "e4m3")])
def test_attend_pages_and_orders(page, layout, dtype, fmt):
    check(build([(1, 130), (5, 97), (70, 200), (0, 0), (200, 333)], 4, 2, 128, page, dtype, fmt,
                layout=layout, seed=page, spare=3))


@pytest.mark.parametrize("n", [1, 7, 150])
def test_attend_shared_prompt(n):
    check(build([(n, 400 + n + 3 * i) for i in range(6)], 4, 2, 128, 16, torch.bfloat16, "i8",
                shared=20, seed=n))


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("reqs", [[(1, 9001)], [(4, 20000), (1, 3)], [(100, 12000)], [(600, 9000)]])
def test_attend_split_over_the_length(reqs, fmt):
    check(build(reqs, 8, 2, 128, 16, torch.bfloat16, fmt, seed=3))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-4, 2.0])
@pytest.mark.parametrize("n", [1, 70])
def test_attend_scales(scale, n):
    check(build([(n, 300)], 4, 2, 128, 16, torch.bfloat16, "i8", seed=1), scale=scale)


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [3, 40, 200])
def test_rows_with_nan_reach_those_that_see_them(n, dtype, fmt):
    """A key or a value held as NaN: rows that see it are NaN, the others are not."""
    from paper_2608_11368_gb300 import binding as B
    kv, D = n + 90, 128
    for which in (1, 3):  # the exponents of keys, of values
        t = build([(n, kv), (n, kv)], 4, 2, D, 16, dtype, fmt, seed=n)
        ref = reference(t, D ** -0.5)
        key = kv - n // 2 - 1  # seen by the later rows of request 0
        at = int(t["table"][0, key // 16]), key % 16
        t["held"][which][at[0], at[1], 1] = 255
        out, _ = B.pair_attend_paged_q8(t["q"], *t["held"], t["table"], t["kv"], t["cu"])
        sees = np.zeros((2 * n, 4), bool)
        sees[key - (kv - n):n, 2:] = True  # query heads 2 and 3 read key head 1
        got = np.isnan(out.double().cpu().numpy())
        assert got[sees].all() and not got[~sees].any()
        err = np.abs(np.where(sees[..., None], 0, out.double().cpu().numpy() - ref[0]))
        assert (err <= 0.02 * ref[2] + 1e-30).all()


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("n", [1, 40])
def test_keys_and_values_of_very_different_sizes(n, fmt):
    """Exponents over their whole range: tiny values beside large ones, zero rows,
    scores of hundreds. Weights are fp32 numbers relative to the largest, which is 1:
    one below 2^-126, the least normal number, may vanish, in the weight itself or in
    a factor that brings a part of the sums to another part's maximum. A key loses
    2 * 2^-126 of its value at most, 500 of them the sum of that; the normaliser is at
    least 1. (Values reach 2^92 times the largest code.)"""
    D = 64
    t = build([(n, 500)], 4, 2, D, 16, torch.bfloat16, fmt, seed=n)
    rng = np.random.default_rng(5)
    ke, ve = t["held"][1], t["held"][3]
    used = (ke != 255).cpu().numpy()
    small = rng.integers(0, 128, used.shape)
    ke.copy_(torch.from_numpy(np.where(used & (rng.random(used.shape) < 0.5), small,
                                       ke.cpu().numpy()).astype(np.uint8)))
    wild = rng.integers(0, 220, used.shape)
    ve.copy_(torch.from_numpy(np.where(used, wild, ve.cpu().numpy()).astype(np.uint8)))
    check(t, lost=500 * 2 * 2.0 ** -126 * 2.0 ** 92 * (127 if fmt == "i8" else 448))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_queries_that_are_rows_of_a_wider_array(dtype):
    t = build([(1, 100), (4, 50), (80, 90)], 4, 2, 64, 16, dtype, "i8", seed=2)
    T = t["q"].shape[0]
    wide = torch.zeros((T, 3, 4, 64), dtype=dtype, device="cuda")
    wide[:, 1] = t["q"]
    t["q"] = wide[:, 1]
    check(t)


def test_more_rows_than_max_new_says():
    t = build([(3, 50), (120, 200)], 4, 2, 128, 16, torch.bfloat16, "e4m3")
    ref = reference(t, 128 ** -0.5)
    for most in (0, 1, 3, 120, 500):
        check(t, ref=ref, max_new=most)


def test_bad_pages_and_lengths_are_reported():
    """A request with a page that does not exist, or a length beyond its table row;
    the others are as they were."""
    from paper_2608_11368_gb300 import binding as B
    for n in (1, 50):
        for what in ("page", "below", "length"):
            t = build([(n, 200), (n, 210), (n, 220)], 4, 2, 128, 16, torch.bfloat16, "i8", seed=n)
            ref = reference(t, 128 ** -0.5)
            if what == "length":
                t["kv"][1] = 10000
            else:
                t["table"][1, 3] = 10 ** 6 if what == "page" else -5
            err = torch.zeros(1, dtype=torch.int32, device="cuda")
            out, _ = B.pair_attend_paged_q8(t["q"], *t["held"], t["table"], t["kv"], t["cu"],
                                            dev_err=err)
            assert B.pair_status_sync(err) == 10
            o = out.double().cpu().numpy()
            for i in (0, 2):
                rows = slice(i * n, (i + 1) * n)
                assert (np.abs(o[rows] - ref[0][rows]) <= 0.02 * ref[2][rows]).all()


@pytest.mark.parametrize("n", [1, 5, 150])
def test_same_results_every_time_on_any_stream_and_captured(n):
    from paper_2608_11368_gb300 import binding as B
    t = build([(n, 2000 + 100 * i) for i in range(9)], 8, 2, 128, 16, torch.bfloat16, "i8", seed=n)

    def call(**kw):
        return B.pair_attend_paged_q8(t["q"], *t["held"], t["table"], t["kv"], t["cu"], max_new=n,
                                      **kw)

    first = [x.clone() for x in call()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(stream=side)
    side.synchronize()
    out, lse = torch.empty_like(first[0]), torch.empty_like(first[1])
    ws = torch.empty(B.pair_attend_workspace_size(9, 8, 2, 128, B.PAIR_BF16), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, lse=lse, ws=ws)
    for fill in (0, 255, 77):  # whatever the workspace holds
        ws.fill_(fill)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    assert torch.equal(other[0], first[0]) and torch.equal(other[1], first[1])


def test_many_requests_and_idle_ones():
    """More requests than a block has threads, most of them with nothing to do."""
    reqs = [(1 if i % 3 == 0 else 0, 1 + i % 40) for i in range(700)]
    check(build(reqs, 4, 4, 64, 8, torch.bfloat16, "e4m3", seed=1), max_new=1)
    check(build(reqs, 4, 2, 64, 8, torch.bfloat16, "i8", seed=2))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(8, 4, 64), (8, 4, 128), (4, 2, 128), (8, 4, 256)])
@pytest.mark.parametrize("n", [1, 6])
def test_one_long_request_among_many(n, heads, dtype):
    """A unit in very many pieces where units are in few on average."""
    reqs = [(n, n + 16 + i % 50) for i in range(130)]
    reqs[33] = (n, 20000)
    Hq, Hkv, D = heads
    check(build(reqs, Hq, Hkv, D, 16, dtype, "i8", seed=n), max_new=n)


def test_exponents_with_strides_of_their_own():
    """Exponent bytes out of a wider array, codes in pages of a larger one."""
    from paper_2608_11368_gb300 import binding as B
    t = build([(1, 100), (6, 77), (90, 190)], 8, 4, 128, 16, torch.bfloat16, "i8", seed=8)
    ref = reference(t, 128 ** -0.5)
    k, ke, v, ve = t["held"]
    wide = torch.full((*ke.shape, 3), 255, dtype=torch.uint8, device="cuda")
    wide[..., 1], wide[..., 2] = ke, ve
    both = torch.zeros((k.shape[0], 2, *k.shape[1:]), dtype=k.dtype, device="cuda")
    both[:, 0], both[:, 1] = k, v
    t["held"] = [both[:, 0], wide[..., 1], both[:, 1], wide[..., 2]]
    assert wide[..., 1].stride(-1) == 3
    check(t, ref=ref)
    assert B.PAIR_CACHE_I8 == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq", [1, 4, 48])
def test_views_with_one_entry(Hq, dtype):
    """Strides over a single page, head or row are not looked at."""
    t = build([(1, 9)], Hq, 1, 64, 16, dtype, "i8", seed=Hq)
    t["q"] = t["q"].as_strided((1, Hq, 64), (Hq * 64 + 1, 64, 1))
    at = int(t["table"][0, 0])
    k, ke, v, ve = (x[at:at + 1] for x in t["held"])
    t["held"] = [k.as_strided((1, 16, 1, 64), (3, 64, 5, 1), k.storage_offset()), ke,
                 v.as_strided((1, 16, 1, 64), (7, 64, 9, 1), v.storage_offset()), ve]
    t["table"].zero_()
    check(t)


def test_a_step_as_it_is_used():
    """Pages, keys and values into the cache in 8 bits, attention over it: the same as
    attention over the values that are read back, to the bounds of both."""
    from paper_2608_11368_gb300 import binding as B
    g = torch.Generator(device="cuda").manual_seed(0)
    R, H, D, page, pages = 5, 4, 128, 16, 200
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for fmt, dt in CODES.items():
        held = [torch.zeros((pages, page, H, D), dtype=dt, device="cuda"),
                torch.zeros((pages, page, H), dtype=torch.uint8, device="cuda")] + [
                    torch.zeros((pages, page, H, D), dtype=dt, device="cuda"),
                    torch.zeros((pages, page, H), dtype=torch.uint8, device="cuda")]
        table = torch.zeros((R, 40), dtype=torch.int32, device="cuda")
        lens, pgs, free, count = i32([0] * R), i32([0] * R), i32(list(range(pages))), i32([pages])
        plain = [torch.zeros((pages, page, H, D), dtype=torch.bfloat16, device="cuda")
                 for _ in "kv"]
        for n in ([200, 3, 0, 17, 64], [1, 1, 0, 1, 1], [4, 4, 1, 0, 40]):
            T = sum(n) + 3
            kv, pgs, cu, slots, taken = B.pair_pages_extend(lens, pgs, i32(n), free, count, table,
                                                            page, T, dev_err=err)
            free, count = torch.roll(free, -int(taken)), count - taken
            q, k, v = (torch.randn((T, h, D), generator=g, device="cuda").bfloat16()
                       for h in (2 * H, H, H))
            B.pair_cache_append_q8(k, v, slots, *held, dev_err=err)
            out, lse = B.pair_attend_paged_q8(q, *held, table, kv, cu, max_new=max(n), dev_err=err)
            back = B.pair_cache_read_q8(slots, *held, dev_err=err)
            B.pair_cache_append(*back, slots, *plain, dev_err=err)
            want, wlse = B.pair_attend_paged(q, *plain, table, kv, cu, max_new=max(n), dev_err=err)
            mag, _ = B.pair_attend_paged(q, plain[0], plain[1].abs(), table, kv, cu, max_new=max(n))
            assert B.pair_status_sync(err) == 0
            # Both sides: weights and output rounded to bf16 (2^-8 of sum p |v| each), and
            # |mag| is itself off by as much.
            bound = 4 * 2.0 ** -8 * 1.02 * mag.float() * (1 + 2.0 ** -6)
            assert ((out.float() - want.float()).abs() <= bound + 1e-30).all()
            same = torch.isinf(wlse)
            assert torch.equal(torch.isinf(lse), same)
            # 2 sides x 2 2^-24 (D size + keys + 16), sizes (scale sum |q_d k_d|) below 16.
            assert ((lse - wlse).abs()[~same] <= 6e-4).all()
            lens = kv


@pytest.mark.parametrize("wide", [False, True])
def test_offsets_beyond_32_bits(wide):
    """Pages more than 4 GiB into the cache, by a page's number or by its stride."""
    from paper_2608_11368_gb300 import binding as B
    H, D, page = 4, 128, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    raw = torch.zeros((1 << 32) + (1 << 26), dtype=torch.int8, device="cuda")
    size = page * H * D
    if wide:  # two pages, 2^32 + 2^15 bytes apart; keys and values side by side
        pages, stride = 2, (1 << 32) + (1 << 15)
        k, v = (raw.as_strided((2, page, H, D), (stride, H * D, D, 1), x * size * 2)
                for x in range(2))
        own = [0, 1]
    else:
        pages = (1 << 32) // size + 100
        k = v = raw[:pages * size].view(pages, page, H, D)
        own = [3, pages - 1]
    ke = torch.full((pages, page, H), 255, dtype=torch.uint8, device="cuda")
    ve = ke if not wide else ke.clone()
    n = 100  # the first page and some of the second
    x = torch.randn((n, H, D), generator=g, device="cuda")
    pos = torch.arange(n, device="cuda")
    slots = torch.tensor(own, device="cuda")[pos // page] * page + pos % page
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.pair_cache_append_q8(x, x, slots, k, ke, v, ve, dev_err=err)
    back, _ = B.pair_cache_read_q8(slots, k, ke, v, ve, dtype=torch.float32, dev_err=err)
    want = rollout.values_q8(*rollout.store_q8(x.double().cpu().numpy(), "i8"))
    assert np.array_equal(back.double().cpu().numpy(), want)
    table = torch.tensor([own], dtype=torch.int32, device="cuda")
    for dtype, rows in ((torch.bfloat16, 1), (torch.bfloat16, 60), (torch.float32, 5)):
        q = torch.randn((rows, 2 * H, D), generator=g, device="cuda").to(dtype)
        out, _ = B.pair_attend_paged_q8(
            q, k, ke, v, ve, table, torch.tensor([n], dtype=torch.int32, device="cuda"),
            torch.tensor([0, rows], dtype=torch.int32, device="cuda"), dev_err=err)
        two = [want.reshape(1, n, H, D)] * 2
        ro, _, mag, _ = rollout.attend_paged(q.double().cpu().numpy(), *two, np.zeros((1, 1), int),
                                             [n], [0, rows], D ** -0.5)
        # Two roundings to bf16 of 2^-8 at most, or sums in fp32.
        rel = 2 * 2.0 ** -8 * 1.02 if dtype == torch.bfloat16 else 2.0 ** -12
        assert (np.abs(out.double().cpu().numpy() - ro) <= rel * mag).all()
    assert B.pair_status_sync(err) == 0
