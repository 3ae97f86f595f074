"""pair_attend_paged against the 64-bit form: single tokens, drafted chunks and
long chunks, head layouts, page sizes, cache orders, rows that see nothing,
whatever lies in places that are not seen.

Error bounds, from the arithmetic. fp32: a score is a dot product of D terms,
off by at most D 2^-24 size (size = scale sum |q_d k_d|); sums over m keys add
m 2^-24, exponentials and rescalings 16 2^-24; relative to mag = sum p |v|
twice (weights and normaliser). bf16: scores as before with twice the unit
(accumulation on the tensor cores need not round to nearest), weights and
output rounded to 8 bits of significand, up to 2^-8 each (the type's unit
roundoff) relative to mag and to |out| <= mag."""
import numpy as np
import pytest
import torch

from oracle import rollout

pytestmark = pytest.mark.gpu


def build(reqs, Hq, Hkv, D, page, dtype, layout="token", seed=0, spare=0, shared=0):
    """Device inputs for requests [(n, kv)]; pages in random order, contents of
    pages that nobody owns and of slots past kv_len NaN."""
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
    k, v = (rng.standard_normal((pages, page, Hkv, D)) for _ in range(2))
    used = np.zeros((pages, page), bool)
    for i, (_, kv) in enumerate(reqs):
        pos = np.arange(kv)
        used[table[i][pos // page], pos % page] = True
    k[~used], v[~used] = np.nan, np.nan
    q = 2.0 * rng.standard_normal((T, Hq, D))

    def dev(x):
        return torch.from_numpy(x).to("cuda").to(dtype)

    def cache(x):
        if layout == "token":
            return dev(x)
        return dev(np.ascontiguousarray(x.transpose(0, 2, 1, 3))).permute(0, 2, 1, 3)

    i32 = lambda x: torch.from_numpy(np.asarray(x, np.int32)).cuda()  # noqa: E731
    return dict(q=dev(q), k=cache(k), v=cache(v), table=i32(table),
                kv=i32([kv for _, kv in reqs]), cu=i32(cu))


def check(t, scale=None, rows=None, **kw):
    from paper_2608_11368_gb300 import binding as B
    D = t["q"].shape[2]
    scale = D ** -0.5 if scale is None else scale
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = B.pair_attend_paged(t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"],
                                   scale=scale, dev_err=err, **kw)
    assert B.pair_status_sync(err) == 0
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    ro, rl, mag, size = rollout.attend_paged(f(t["q"]), f(t["k"]), f(t["v"]),
                                             t["table"].cpu().numpy(), t["kv"].cpu().numpy(),
                                             t["cu"].cpu().numpy(), scale)
    out, lse = f(out), f(lse)
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
    assert (np.abs(out - ro)[fin] <= (rel[..., None] * mag)[fin] + 1e-30).all()
    return out, lse_all


SHAPES = {
    "token": [(1, 1)],
    "tokens": [(1, 1), (1, 15), (1, 16), (1, 17), (1, 63), (1, 64), (1, 65), (1, 700)],
    "drafts": [(5, 5), (5, 64), (3, 130), (8, 8), (2, 1000), (5, 257)],
    "chunk": [(40, 40), (129, 300), (1, 77), (64, 64)],
    "long": [(300, 700), (257, 257)],
    "none": [(0, 0), (0, 33), (4, 2), (1, 0), (3, 3), (0, 5), (130, 7)],
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (3, 3, 128), (10, 2, 64), (2, 1, 256)])
@pytest.mark.parametrize("what", sorted(SHAPES))
def test_attend(what, heads, dtype):
    Hq, Hkv, D = heads
    check(build(SHAPES[what], Hq, Hkv, D, 16, dtype, seed=len(what)))


@pytest.mark.parametrize("page", [1, 5, 8, 24, 32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["token", "head"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_pages_and_orders(page, layout, dtype):
    check(build([(1, 130), (5, 97), (70, 200), (0, 0), (200, 333)], 4, 2, 128, page, dtype,
                layout=layout, seed=page, spare=3))


@pytest.mark.parametrize("n", [1, 7, 150])
def test_attend_shared_prompt(n):
    check(build([(n, 400 + n + 3 * i) for i in range(6)], 4, 2, 128, 16, torch.bfloat16, shared=20,
                seed=n))


@pytest.mark.parametrize("reqs", [[(1, 9001)], [(4, 20000), (1, 3)], [(100, 12000)], [(600, 9000)]])
def test_attend_long_keys_few_rows(reqs):
    """One long request is cut over many CTAs and joined."""
    check(build(reqs, 2, 1, 128, 16, torch.bfloat16, seed=5))
    check(build(reqs[:1], 2, 1, 64, 16, torch.bfloat16, seed=6))


def test_attend_many_requests():
    rng = np.random.default_rng(3)
    reqs = [(int(rng.integers(0, 3)), int(rng.integers(3, 90))) for _ in range(3000)]
    check(build(reqs, 2, 1, 64, 16, torch.bfloat16, seed=3))


@pytest.mark.parametrize("D", [64, 128])
def test_attend_many_short_chunks(D):
    """Hundreds of short chunks, some of one tile of rows, some of more, so that
    a CTA works off many units of few key tiles one after the other."""
    rng = np.random.default_rng(D)
    reqs = [(int(n), int(n + rng.integers(0, 200))) for n in rng.integers(0, 130, 400)]
    check(build(reqs, 4, 2, D, 32, torch.bfloat16, seed=D))
    reqs = [(int(n), int(n + rng.integers(0, 140))) for n in rng.integers(130, 270, 60)]
    check(build(reqs, 10, 2, D, 8, torch.bfloat16, layout="head", seed=D + 1))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n", [6, 150])
def test_attend_what_a_row_does_not_see(n, bad, dtype):
    """A later token's key and value are not finite: earlier rows do not
    change, the rows that see it take it as the sum does."""
    t = build([(n, 200 + n), (2, 50)], 4, 2, 128, 16, dtype, seed=9)
    want, _ = check(t)
    pos = 200 + n - 2  # seen by the last two rows of the chunk
    pg, off = int(t["table"][0, pos // 16]), pos % 16
    t["v"][pg, off, 1, 3] = bad
    from paper_2608_11368_gb300 import binding as B
    out, _ = B.pair_attend_paged(t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"])
    out = out.double().cpu().numpy()
    hit = np.zeros(out.shape, bool)
    hit[n - 2:n, 2:4, 3] = True
    assert (out[~hit] == want[~hit]).all()
    assert not np.isfinite(out[hit]).any()
    if bad == float("inf"):
        assert (out[hit] == np.inf).all()
    t["k"][pg, off, 0, 5] = float("nan")
    out, lse = B.pair_attend_paged(t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"])
    out, lse = out.double().cpu().numpy(), lse.cpu().numpy()
    assert np.isnan(out[n - 2:n, :2]).all() and np.isnan(lse[n - 2:n, :2]).all()
    assert (out[:n - 2] == want[:n - 2]).all()


@pytest.mark.parametrize("n", [1, 5, 90])
def test_attend_strided_queries_and_scale(n):
    t = build([(n, 300), (n, n)], 6, 2, 64, 16, torch.bfloat16, seed=2)
    T = t["q"].shape[0]
    wide = torch.full((T, 10, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:8] = t["q"]
    t["q"] = wide[:, 2:8]
    for scale in (0.3, -0.2, 0.0, 3.0):
        check(t, scale=scale)


@pytest.mark.parametrize("n", [1, 90])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attend_output_on_a_16_byte_boundary(n, dtype):
    t = build([(n, 300), (2 * n, 2 * n)], 4, 2, 128, 16, dtype, seed=4)
    shape = t["q"].shape
    out = torch.empty(t["q"].numel() + 8, dtype=dtype, device="cuda")[8:].view(shape)
    assert out.data_ptr() % 32 == (16 if dtype is torch.bfloat16 else 0)
    check(t, out=out)


@pytest.mark.parametrize("n", [1, 3, 140])
def test_attend_large_scores(n):
    """Scores far apart: weights that vanish, maxima that move in every tile."""
    t = build([(n, 513)], 4, 1, 128, 16, torch.bfloat16, seed=8)
    t["k"] *= torch.linspace(0.1, 9.0, t["k"].shape[0], device="cuda").to(torch.bfloat16)[:, None,
                                                                                       None, None]
    check(t)


def test_attend_cache_beyond_32_bit_offsets():
    """Pages whose element offsets pass 2^31 (a view of 4.3 GB and more)."""
    pages, page, Hkv, D = 70000, 16, 16, 128
    try:
        k = torch.empty((pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
        v = torch.empty((pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
    except torch.cuda.OutOfMemoryError:
        pytest.skip("no room")
    assert k.numel() > 2 ** 31
    for n, kv in ((1, 90), (140, 200)):
        t = build([(n, kv)], 16, 16, 128, 16, torch.bfloat16, seed=n)
        m = t["k"].shape[0]
        k[-m:], v[-m:] = t["k"], t["v"]
        from paper_2608_11368_gb300 import binding as B
        want = B.pair_attend_paged(t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"])
        got = B.pair_attend_paged(t["q"], k, v, t["table"] + (pages - m), t["kv"], t["cu"])
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


@pytest.mark.parametrize("n", [1, 6, 200])
def test_attend_repeats_bit_for_bit_and_on_another_stream(n):
    from paper_2608_11368_gb300 import binding as B
    t = build([(n, 2000), (n, 900), (1, 31)], 8, 2, 128, 16, torch.bfloat16, seed=1)
    args = (t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"])
    a = B.pair_attend_paged(*args)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = B.pair_attend_paged(*args)
    c = B.pair_attend_paged(*args, stream=s)
    s.synchronize()
    for x in (b, c):
        assert torch.equal(a[0], x[0]) and torch.equal(a[1], x[1])


def test_attend_reports_pages_that_do_not_fit():
    from paper_2608_11368_gb300 import binding as B
    t = build([(2, 40), (2, 40)], 4, 2, 64, 16, torch.bfloat16)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def status(**change):
        x = dict(t, **change)
        out, _ = B.pair_attend_paged(x["q"], x["k"], x["v"], x["table"], x["kv"], x["cu"],
                                     dev_err=err)
        st = B.pair_status_sync(err)
        return st, out

    st, good = status()
    assert st == 0
    for page in (-1, t["k"].shape[0], 2 ** 31 - 1, -2 ** 31):
        bad = t["table"].clone()
        bad[1, 1] = page
        st, out = status(table=bad)
        assert B.STATUS_NAMES[st] == "PAIR_ERR_PAGES"
        assert torch.equal(out[:2], good[:2])
    for kv in ([40, -1], [40, 49], [40, 2 ** 31 - 1]):
        st, out = status(kv=torch.tensor(kv, dtype=torch.int32, device="cuda"))
        assert B.STATUS_NAMES[st] == "PAIR_ERR_PAGES"
        assert torch.equal(out[:2], good[:2])
    for cu in ([0, 2, 1], [0, 2, 5], [0, 2, 2 ** 31 - 1], [0, -2, 4]):
        st, out = status(cu=torch.tensor(cu, dtype=torch.int32, device="cuda"))
        assert B.STATUS_NAMES[st] == "PAIR_ERR_PAGES"


def test_attend_reports_lengths_that_pass_32_bits():
    """A table row of 2^31 tokens: a length that leaves no room for whole tiles
    in 32 bits is reported, and the other request is served."""
    from paper_2608_11368_gb300 import binding as B
    for dtype in (torch.bfloat16, torch.float32):
        t = build([(2, 40), (2, 40)], 4, 2, 64, 64, dtype)
        x = {c: t[c][int(t["table"][0, 0]):, :1][:1].expand(1, 2 ** 30, 2, 64) for c in "kv"}
        table = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")

        def run(kv):
            kv = torch.tensor(kv, dtype=torch.int32, device="cuda")
            out, _ = B.pair_attend_paged(t["q"], x["k"], x["v"], table, kv, t["cu"], dev_err=err)
            return B.pair_status_sync(err), out

        st, good = run([40, 40])
        assert st == 0 and bool(torch.isfinite(good).all())
        for kv in (2 ** 31 - 1, 2 ** 31 - 4096):
            st, out = run([40, kv])
            assert B.STATUS_NAMES[st] == "PAIR_ERR_PAGES"
            assert torch.equal(out[:2], good[:2])


def test_attend_refuses():
    from paper_2608_11368_gb300 import binding as B
    t = build([(2, 40)], 4, 2, 64, 16, torch.bfloat16)
    args = [t["q"], t["k"], t["v"], t["table"], t["kv"], t["cu"]]

    def refuses(kind, i=None, x=None, **kw):
        a = list(args)
        if i is not None:
            a[i] = x
        with pytest.raises(kind):
            B.pair_attend_paged(*a, **kw)

    refuses(TypeError, 0, t["q"].half())
    refuses(TypeError, 0, t["q"].cpu())
    refuses(TypeError, 1, t["k"].float())
    refuses(ValueError, 2, t["v"][:, :8])
    refuses(ValueError, 1, t["k"][0])
    refuses(TypeError, 3, t["table"].long())
    refuses(ValueError, 4, t["kv"][:0])
    refuses(ValueError, 5, t["cu"][:1])
    refuses(ValueError, 0, t["q"][:, :, :32])
    refuses(B.PairError, 0, t["q"][:, :3].contiguous())              # heads do not divide
    refuses(B.PairError, ws=torch.empty(512, dtype=torch.uint8, device="cuda"))
    refuses(B.PairError, scale=float("nan"))
    odd = torch.zeros(2 * 4 * 65, dtype=torch.bfloat16, device="cuda")
    refuses(B.PairError, 0, odd[1:513].view(2, 4, 64))               # 2-byte aligned
    refuses(B.PairError, 0, odd.view(2, 4, 65)[:, :, :64])           # stride of 65 elements
    t96 = build([(2, 40)], 4, 2, 96, 16, torch.bfloat16)
    with pytest.raises(B.PairError) as e:
        B.pair_attend_paged(*(t96[k] for k in ("q", "k", "v", "table", "kv", "cu")))
    assert B.STATUS_NAMES[e.value.status] == "PAIR_ERR_UNSUPPORTED"
