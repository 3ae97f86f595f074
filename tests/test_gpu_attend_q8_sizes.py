"""pair_attend_paged_q8 over rows of extreme sizes, each key head's against its own bounds,
so that large numbers do not hide what happens to small ones: every row of a key head has
the same exponent byte, from the least to the largest, on one side (keys or values), in
the kernels for few rows and for many.

The bounds, from the header's text. A score is a dot product of D terms, off by D 2^-24
size (size = scale sum |q_d k_d|, twice that for bf16, whose sums on the tensor cores need
not round to nearest); sums over m keys add m 2^-24, exponentials and rescalings 16 2^-24;
relative to mag = sum p |v| twice (weights and normaliser). bf16: weights and output rounded
once each, 2^-8 of mag. What is tiny: with few rows a weight times the value's power of two
is a bf16 number (fp32 queries: the last of three is), so it is off by 2^-134 below 2^-126,
or vanishes: c min(2^-134 / L, p 2^(b - 127)) for the code c of a key with the weight p, L >= 1
the sum of the weights relative to the largest. With many rows a stored number over 2^8 is
a bf16 number: it is off by 2^-126 if its last place is below 2^-125, which whole numbers' are
for b < 2 and e4m3's for b < 11. An output below bf16's normal numbers is off by 2^-134."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

CODES = {"i8": torch.int8, "e4m3": torch.float8_e4m3fn}
ORDINARY, KV, PAGE, GROUP = 122, 300, 16, 2


def inputs(fmt, D, n, keys, values, dtype):
    """One request of n rows over KV keys; a byte for each key head's keys, and values.
    Queries make up for the keys' size. Codes over their whole range, ordinary ones."""
    rng = np.random.default_rng(len(keys) + n + D)
    pages, Hkv = -(-KV // PAGE), len(keys)
    codes = []
    for _ in "kv":
        x = rng.standard_normal((pages, PAGE, Hkv, D))
        if fmt == "i8":
            x = np.clip(np.rint(30 * x), -127, 127)
        codes.append(torch.from_numpy(np.clip((1 if fmt == "i8" else 120) * x, -448, 448)).to(
            CODES[fmt]))
    exps = [np.broadcast_to(np.array(b, np.uint8), (pages, PAGE, Hkv)).copy()
            for b in (keys, values)]
    q = rng.standard_normal((n, Hkv, GROUP, D)) * (2.0 if fmt == "i8" else 0.5)
    q *= 2.0 ** (ORDINARY - np.array(keys, np.float64))[:, None, None]
    q = torch.from_numpy(q.reshape(n, Hkv * GROUP, D)).to(dtype)
    return q, codes, exps


def bounds(q, codes, exps, n, many, D, fmt, keys, values):
    """out, lse, their bounds, mag: [n, Hkv, GROUP, ..] in 64 bits."""
    f32 = q.dtype == torch.float32
    Hkv = len(keys)
    c = [x.to(torch.float32).double().numpy().reshape(-1, Hkv, D)[:KV] for x in codes]
    k, v = (y * 2.0 ** (np.array(b, np.float64) - 127)[:, None] for y, b in zip(c, (keys, values)))
    x, scale = q.double().numpy().reshape(n, Hkv, GROUP, D), D ** -0.5
    s = scale * np.einsum("nhgd,khd->nhgk", x, k)
    size = scale * np.einsum("nhgd,khd->nhgk", np.abs(x), np.abs(k))
    unseen = np.arange(KV)[None] > (KV - n + np.arange(n))[:, None]
    s[np.broadcast_to(unseen[:, None, None], s.shape)] = -np.inf
    size[np.isinf(s)] = 0.0
    top = s.max(-1, keepdims=True)
    w = np.exp(s - top)
    total = w.sum(-1, keepdims=True)
    p, lse = w / total, (top + np.log(total))[..., 0]
    out = np.einsum("nhgk,khd->nhgd", p, v)
    mag = np.einsum("nhgk,khd->nhgd", p, np.abs(v))
    sums = (1.0 if f32 else 2.0) * 2.0 ** -24 * (D * size.max(-1) + KV + 16)
    unit = 2.0 ** (np.array(values, np.float64) - 127)[:, None, None]
    last = 2 if fmt == "i8" else 11
    if many:
        off = (np.array(keys) < last)[:, None] * 2.0 ** -126
        sums += scale * np.abs(x).sum(-1) * off
        lost = (np.array(values) < last)[:, None, None] * 2.0 ** -126
    else:
        lost = np.einsum("nhgk,khd->nhgd", np.minimum(p * unit, 2.0 ** -134 / total), np.abs(c[1]))
    rel = 2 * sums + (0.0 if f32 else 2 * 2.0 ** -8 * 1.01)
    out_bound = rel[..., None] * mag + lost + (0.0 if f32 else 2.0 ** -134)
    return out, lse, out_bound, sums + 2.0 ** -22 * np.abs(lse), mag


def check(fmt, D, n, keys, values, dtype):
    from paper_2608_11368_gb300 import binding as B
    q, codes, exps = inputs(fmt, D, n, keys, values, dtype)
    many = dtype == torch.bfloat16 and D <= 128 and n * GROUP > 32
    want, lse_want, bound, lse_bound, mag = bounds(q, codes, exps, n, many, D, fmt, keys, values)
    # The bounds say something: a factor of two would be outside.
    assert (np.median(bound / mag, axis=(0, 2, 3)) < 0.4).all()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kc, vc = (x.cuda() for x in codes)
    ke, ve = (torch.from_numpy(x).cuda() for x in exps)
    err = i32([0])
    table = torch.arange(kc.shape[0], dtype=torch.int32, device="cuda")[None].contiguous()
    out, lse = B.pair_attend_paged_q8(q.cuda(), kc, ke, vc, ve, table, i32([KV]), i32([0, n]),
                                      dev_err=err)
    assert B.pair_status_sync(err) == 0
    out = out.double().cpu().numpy().reshape(want.shape)
    lse = lse.double().cpu().numpy().reshape(lse_want.shape)
    assert (np.abs(lse - lse_want) <= lse_bound).all()
    assert (np.abs(out - want) <= bound).all()


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 12, 16, 100])
@pytest.mark.parametrize("values", [(0, 1, 2, 10), (20, 129, 142), (130, 143, 200, 216)])
def test_values_of_every_size(values, n, D, dtype, fmt):
    check(fmt, D, n, (ORDINARY,) * len(values), values, dtype)


@pytest.mark.parametrize("fmt", sorted(CODES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [1, 12, 16, 100])
@pytest.mark.parametrize("keys", [(2, 10, 11, 60), (20, 129, 142), (130, 143, 200, 240)])
def test_keys_of_every_size(keys, n, D, dtype, fmt):
    """Large keys under queries that are as small: a score is what it is, although a product
    of codes and the key's power of two alone would leave fp32's range."""
    check(fmt, D, n, keys, (ORDINARY,) * len(keys), dtype)


@pytest.mark.parametrize("dtype,D,page,rows,names", [
    (torch.bfloat16, 128, 16, 100, ["attend_q8_many"]),
    (torch.bfloat16, 64, 8, 33, ["attend_q8_many"]),
    (torch.bfloat16, 128, 16, 32, ["attend_q8_few"]),
    (torch.bfloat16, 128, 12, 100, ["attend_q8_few"]),
    (torch.bfloat16, 256, 16, 100, ["attend_q8_few"]),
    (torch.float32, 128, 16, 100, ["attend_q8_few"])])
def test_which_kernel_a_chunk_goes_to(dtype, D, page, rows, names):
    """As the header says it: by the type, the head size, the pages and the rows per key
    head; a chunk that is alone has one launch and the joining pass."""
    from paper_2608_11368_gb300 import binding as B
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pages = -(-KV // page)
    codes = torch.zeros((pages, page, 1, D), dtype=torch.int8, device="cuda")
    exps = torch.zeros((pages, page, 1), dtype=torch.uint8, device="cuda")
    q, err = torch.zeros((rows, 1, D), dtype=dtype, device="cuda"), i32([0])
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous()
    B.pair_timing_enable(True)
    try:
        B.pair_attend_paged_q8(q, codes, exps, codes, exps, table, i32([KV]), i32([0, rows]),
                               dev_err=err)
        got = [n for n, _ in B.pair_timing_read()]
    finally:
        B.pair_timing_enable(False)
    assert B.pair_status_sync(err) == 0
    assert got == [*names, "attend_join"]
