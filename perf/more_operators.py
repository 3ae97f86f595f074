"""Operators of a rollout cache held in 8 bits, as timed cases.

A step of generating the continued rollouts writes its chunk's keys and values
into the paged cache in 8 bits (pair_cache_append_q8), attends over that cache
(pair_attend_paged_q8), and whoever wants the stored values again (a trainer
that scores a prefix, another cache) reads them back (pair_cache_read_q8).

The stored form. A row of the D entries of one token and head is held as codes
c and one exponent byte b, and stands for c 2^(b - 127): c are whole numbers
of -127 to 127 ("i8") or e4m3 floating-point numbers ("e4m3"). The exponent
is the least one, not below -127, with which the row's largest entry does not
round beyond the largest code, 127 or 448; codes are rounded to nearest even.

The plain forms are elementary torch operations in 32 bits over requests of
similar lengths at a time; a scheduler's host copy of the lengths is part of
the state. `exact` computes the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # One rollout generating token by token: 16 query and 8 key heads of
        # 128 over a few hundred cached tokens. Latency is all there is.
        dict(name="attend_1x1", kind="attend", fmt="i8", dtype="bf16", B=1, G=1, hq=16, hkv=8,
             D=128, page=16, prompt=0, dist="uniform", ctx_lo=700, ctx_hi=700, n_lo=1, n_hi=1,
             layout="token"),
        # 8 prompts x 8 rollouts of 256 to 2048 tokens, a token each.
        dict(name="attend_8x8_token", kind="attend", fmt="e4m3", dtype="bf16", B=8, G=8, hq=16,
             hkv=8, D=128, page=16, prompt=192, dist="uniform", ctx_lo=256, ctx_hi=2048, n_lo=1,
             n_hi=1, layout="head"),
        # 16 x 16 rollouts of 512 to 4096 tokens on 32/8 heads, each with
        # four drafted tokens behind its last one.
        dict(name="attend_16x16_drafts", kind="attend", fmt="i8", dtype="bf16", B=16, G=16, hq=32,
             hkv=8, D=128, page=32, prompt=512, dist="uniform", ctx_lo=512, ctx_hi=4096, n_lo=5,
             n_hi=5, layout="token"),
        # The heavy-tailed workload: 32 x 16 rollouts, median 1500 tokens,
        # capped at 16384, a token each: the most bytes one call reads.
        dict(name="attend_32x16_skew", kind="attend", fmt="i8", dtype="bf16", B=32, G=16, hq=16,
             hkv=8, D=128, page=64, prompt=256, dist="lognormal", ctx_lo=1500, ctx_hi=16384,
             n_lo=1, n_hi=1, layout="token"),
        # The same with 4-bit significands, by head.
        dict(name="attend_32x16_skew_e4m3", kind="attend", fmt="e4m3", dtype="bf16", B=32, G=16,
             hq=32, hkv=8, D=128, page=64, prompt=256, dist="lognormal", ctx_lo=1500, ctx_hi=16384,
             n_lo=1, n_hi=1, layout="head"),
        # Chunks of prompts and of continued prefixes scored at once: ragged
        # chunks of up to 2048 tokens behind up to 6144 cached ones.
        dict(name="attend_chunks_4", kind="attend", fmt="i8", dtype="bf16", B=4, G=1, hq=32, hkv=8,
             D=128, page=16, prompt=0, dist="uniform", ctx_lo=1000, ctx_hi=6144, n_lo=1025,
             n_hi=2048, layout="token"),
        # Prompts' pieces of up to 256 tokens behind short prefixes.
        dict(name="attend_chunks_64_e4m3", kind="attend", fmt="e4m3", dtype="bf16", B=64, G=1,
             hq=16, hkv=8, D=128, page=16, prompt=0, dist="uniform", ctx_lo=100, ctx_hi=2048,
             n_lo=32, n_hi=256, layout="token"),
        # The fp32 reference head's 4 x 8 rollouts, heads of 64, pages of 24.
        dict(name="attend_f32_4x8", kind="attend", fmt="i8", dtype="f32", B=4, G=8, hq=4, hkv=2,
             D=64, page=24, prompt=0, dist="uniform", ctx_lo=32, ctx_hi=640, n_lo=3, n_hi=3,
             layout="token"),
        # New keys and values of 64 tokens stored and read back as they are
        # held, and of four chunks of 2048.
        dict(name="store_64", kind="store", fmt="i8", dtype="bf16", T=64, hkv=8, D=128, page=16,
             pages=4096, layout="token"),
        dict(name="store_8192_e4m3", kind="store", fmt="e4m3", dtype="bf16", T=8192, hkv=8, D=128,
             page=16, pages=4096, layout="head"),
        # A rollout's prefix read back, and the prefixes of a batch.
        dict(name="read_700", kind="read", fmt="e4m3", dtype="f32", T=700, hkv=8, D=128, page=16,
             pages=4096, layout="token"),
        dict(name="read_65536", kind="read", fmt="i8", dtype="bf16", T=65536, hkv=8, D=128, page=16,
             pages=8192, layout="token"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "attend", "attend", "store", "read"))
    layout, fmt = rng.choice(("token", "head")), rng.choice(("i8", "e4m3"))
    if kind != "attend":
        hkv, D = rng.choice((1, 2, 4, 8)), rng.choice((64, 80, 128, 128, 256))
        page = rng.choice((8, 16, 24, 64))
        T = _log_int(rng, 1, 8192 if kind == "store" else 32768)
        return dict(kind=kind, fmt=fmt, dtype=rng.choice(("bf16", "bf16", "f32")), T=T, hkv=hkv,
                    D=D, page=page, pages=8192, layout=layout)
    f32 = rng.random() < 0.2
    hq, hkv = rng.choice(((16, 8), (32, 8), (8, 8), (4, 1), (6, 2), (15, 3), (16, 1)))
    c = dict(kind=kind, fmt=fmt, dtype="f32" if f32 else "bf16", G=rng.choice((1, 4, 8, 16)), hq=hq,
             hkv=hkv, D=rng.choice((64, 128, 128, 128, 256) if not f32 else (64, 128)),
             page=rng.choice((8, 16, 16, 32, 64, 128, 24)))
    n_hi = rng.choice((1, rng.randint(2, 8), _log_int(rng, 9, 2048)))
    n_lo = rng.choice((n_hi, n_hi // 2, 0)) if n_hi > 1 else 1
    skew = rng.random() < 0.25
    ctx_hi = _log_int(rng, 16, 16384 if not f32 else 1024)
    ctx_lo = max(1, ctx_hi // 8) if skew else rng.choice((0, ctx_hi // 2, ctx_hi))
    mean = (ctx_lo * 1.5 if skew else (ctx_lo + ctx_hi) / 2) + n_hi
    most_bytes = 2.0e9 if not f32 else 5.0e7
    most_flops = 3.5e11 if not f32 else 2e10
    R = min(512, most_bytes / (2 * hkv * c["D"] * mean),
            most_flops / (4.0 * hq * c["D"] * n_hi * mean))
    R = _log_int(rng, 1, max(1, int(R)))
    c["G"] = min(c["G"], R)
    c["B"] = max(1, R // c["G"])
    prompt = 0
    if c["G"] > 1 and rng.random() < 0.5:
        prompt = min(ctx_lo, ctx_hi // 2) // c["page"] * c["page"]
    c.update(prompt=prompt, dist="lognormal" if skew else "uniform", ctx_lo=ctx_lo, ctx_hi=ctx_hi,
             n_lo=n_lo, n_hi=n_hi, layout=layout)
    return c


# ----------------------------------------------------------------- inputs
def _lib():
    from paper_2608_11368_gb300 import binding
    return binding


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _ints(rng, lo, hi, n):
    return rng.integers(lo, hi, size=n, endpoint=True).astype(np.int64)


def _chunks(rng, lo, hi, n):
    """n lengths in [lo, hi] whose sum does not depend on the draw: a step's
    arrays have a capacity."""
    x = _ints(rng, lo, hi, n)
    off = min(max(1, n * (lo + hi) // 2), n * hi) - int(x.sum())
    for i in rng.permutation(n):  # what is missing or too much, from requests in no order
        step = min(off, hi - x[i]) if off > 0 else max(off, lo - x[i])
        x[i] += step
        off -= step
    return x


def _contexts(case, rng, n):
    if case["dist"] == "lognormal":  # ctx_lo is the median, ctx_hi the cap
        x = np.rint(np.exp(math.log(case["ctx_lo"]) + 0.9 * rng.standard_normal(n)))
        return np.clip(x, max(1, case["prompt"]), case["ctx_hi"]).astype(np.int64)
    return np.maximum(_ints(rng, case["ctx_lo"], case["ctx_hi"], n), case["prompt"])


def _gains(case, g, keys):
    """Sizes of the D channels of every head: keys have a few channels that are
    far larger than the others, values hardly."""
    x = torch.exp((0.6 if keys else 0.15) * torch.randn((case["hkv"], case["D"]), generator=g,
                                                       device=DEV))
    return x / x.square().mean(-1, keepdim=True).sqrt()


def _power(b):
    """2^(b - 127) for whole numbers 0 <= b <= 254, by its bits."""
    return torch.where(b > 0, b.int() << 23, 1 << 22).view(torch.float32)


def _quantised(x, fmt):
    """Codes and exponent bytes of rows [.., D] in fp32."""
    top = x.abs().amax(-1)
    f, e = torch.frexp(top)  # top = f 2^e, f in [0.5, 1)
    # The largest code and half a step: what is below rounds to it at most.
    most, bits = (127.5, 7) if fmt == "i8" else (464.0, 9)
    e = torch.where(f * 2.0 ** bits < most, e - bits, e - bits + 1)
    e = torch.where(top > 0, e, -127).clamp_min(-127)
    y = x * _power(127 - e)[..., None]
    c = y.round().to(torch.int8) if fmt == "i8" else y.to(torch.float8_e4m3fn)
    return c, (e + 127).to(torch.uint8)


def _values(c, b):
    """What codes and exponent bytes stand for, in fp32."""
    return c.float() * _power(b)[..., None]


def _take(c, at):
    """Rows of codes, by whole bytes: not every indexing takes 8-bit
    floating-point numbers."""
    return c.view(torch.uint8)[at].view(c.dtype)


def _cache(case, g, pages, keys):
    """A filled cache: codes [pages, page, hkv, D], exponents [pages, page, hkv],
    laid out by token or by head."""
    page, hkv, D = case["page"], case["hkv"], case["D"]
    head = case["layout"] == "head"
    shape = (pages, hkv, page, D) if head else (pages, page, hkv, D)
    c = torch.empty(shape, dtype=torch.int8 if case["fmt"] == "i8" else torch.float8_e4m3fn,
                    device=DEV)
    b = torch.empty(shape[:3], dtype=torch.uint8, device=DEV)
    gains = _gains(case, g, keys)
    gains = gains[:, None] if head else gains
    step = max(1, (1 << 26) // (page * hkv * D))
    for a in range(0, pages, step):
        x = torch.randn((min(step, pages - a),) + shape[1:], generator=g, device=DEV) * gains
        # Tokens differ in size, some by far.
        x *= torch.exp(0.5 * torch.randn(x.shape[:3] + (1,), generator=g, device=DEV))
        c[a:a + step], b[a:a + step] = _quantised(x, case["fmt"])
    return (c.permute(0, 2, 1, 3), b.permute(0, 2, 1)) if head else (c, b)


def _alike(kv, n, per_key, per_pair):
    """Requests in runs of similar lengths, padded to the longest of each, whose
    padded keys and scores stay within half a gigabyte or so in fp32."""
    runs, run = [], []
    for i in np.argsort(kv, kind="stable"):
        if n[i] == 0 or kv[i] == 0:
            continue
        wide = max([n[i]] + [n[j] for j in run])
        if run and (len(run) + 1) * kv[i] * (per_key + per_pair * wide) > 1 << 27:
            runs.append(run)
            run = []
        run.append(int(i))
    return runs + [run] if run else runs


def _prepare_attend(case, seed):
    rng, g = np.random.default_rng(int(seed)), _gen(seed)
    R, page, shared = case["B"] * case["G"], case["page"], case["prompt"] // case["page"]
    ctx = _contexts(case, rng, R)
    n = _chunks(rng, case["n_lo"], case["n_hi"], R)
    kv = ctx + n
    need = -(-kv // page)
    own_pages = np.maximum(need - shared, 0)
    total = int(case["B"] * shared + own_pages.sum())
    width = max(1, int(need.max()))
    pages = total + 3
    order = rng.permutation(pages).astype(np.int32)  # pages come in no order
    table = np.zeros((R, width), np.int32)
    at = case["B"] * shared
    for i in range(R):
        b = i // case["G"]
        table[i, :shared] = order[b * shared:(b + 1) * shared]
        table[i, shared:need[i]] = order[at:at + own_pages[i]]
        at += int(own_pages[i])
    cu = np.concatenate([[0], np.cumsum(n)])
    T = int(cu[-1])
    dt = _dtype(case)
    # Normalised heads give scores of a few units either way.
    q = (2.0 * torch.randn((T, case["hq"], case["D"]), generator=g, device=DEV)).to(dt)
    k, ke = _cache(case, g, pages, True)
    v, ve = _cache(case, g, pages, False)
    runs = [(torch.tensor(r, device=DEV), int(max(kv[i] for i in r)), int(max(n[i] for i in r)))
            for r in _alike(kv, n, case["hkv"] * case["D"], case["hq"])]
    s = dict(case=case, runs=runs, kv_host=kv.tolist(), cu_host=cu.tolist(), q=q, k=k, ke=ke, v=v,
             ve=ve, table=torch.from_numpy(table).to(DEV),
             kv=torch.from_numpy(kv.astype(np.int32)).to(DEV),
             cu=torch.from_numpy(cu.astype(np.int32)).to(DEV), scale=case["D"] ** -0.5)
    if own:
        L = _lib()
        s["out"] = torch.empty_like(q)
        s["lse"] = torch.empty((T, case["hq"]), dtype=torch.float32, device=DEV)
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        need_b = L.pair_attend_workspace_size(R, case["hq"], case["hkv"], case["D"],
                                              L.PAIR_BF16 if dt == torch.bfloat16 else L.PAIR_F32)
        s["ws"] = torch.empty(max(need_b, 256), dtype=torch.uint8, device=DEV)
    return s


def _prepare_rows(case, seed):
    """New tokens in chunks of 64 whose pages come in no order; some rows are
    spare."""
    g = _gen(seed)
    T, page, pages, dt = case["T"], case["page"], case["pages"], _dtype(case)
    chunk = 64
    rows = -(-chunk // page)
    n_chunks = -(-T // chunk)
    order = torch.randperm(pages, generator=g, device=DEV)[:n_chunks * rows].view(n_chunks, rows)
    t = torch.arange(T, device=DEV)
    pos = t % chunk
    slots = order[t // chunk, pos // page] * page + pos % page
    slots = torch.where(torch.rand(T, generator=g, device=DEV) < 0.02, -1, slots)
    k, ke = _cache(case, g, pages, True)
    v, ve = _cache(case, g, pages, False)
    s = dict(case=case, slots=slots.to(torch.int64), k=k, ke=ke, v=v, ve=ve)
    if case["kind"] == "store":
        # Keys and values as one projection leaves them: rows of both, strided.
        kv = torch.randn((T, 2, case["hkv"], case["D"]), generator=g, device=DEV)
        kv[:, 0] *= _gains(case, g, True)
        s["k_new"], s["v_new"] = kv.to(dt)[:, 0], kv.to(dt)[:, 1]
    if own:
        shape = (T, case["hkv"], case["D"])
        s["k_out"], s["v_out"] = (torch.empty(shape, dtype=dt, device=DEV) for _ in "kv")
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    return (_prepare_attend if case["kind"] == "attend" else _prepare_rows)(case, seed)


# ------------------------------------------------------------------ one pass
def _plain_attend(s):
    c = s["case"]
    hq, hkv, D, page = c["hq"], c["hkv"], c["D"], c["page"]
    g = hq // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float32, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, device=DEV)
    for i, m, n in s["runs"]:
        kv, first = s["kv"][i].long(), s["cu"][i].long()
        new = s["cu"][i + 1].long() - first
        key, row = torch.arange(m, device=DEV), torch.arange(n, device=DEV)
        where = s["table"][i[:, None], key // page].long()
        where = torch.where(key < kv[:, None], where, 0)
        at = (where, key % page)
        k, v = _values(_take(s["k"], at), s["ke"][at]), _values(_take(s["v"], at), s["ve"][at])
        there = row < new[:, None]
        rows = (first[:, None] + torch.where(there, row, 0))
        q = s["q"][rows].float().view(-1, n, hkv, g, D).permute(0, 2, 3, 1, 4)
        sc = torch.matmul(q.reshape(-1, hkv, g * n, D), k.permute(0, 2, 3, 1))
        sc = (sc * s["scale"]).view(-1, hkv, g, n, m)
        seen = key <= (kv - new)[:, None, None] + row[:, None]
        sc.masked_fill_(~seen[:, None, None], -math.inf)
        mx = sc.amax(-1, keepdim=True)
        sc.sub_(torch.where(mx == -math.inf, 0.0, mx)).exp_()
        tot = sc.sum(-1, keepdim=True)
        o = torch.matmul(sc.view(-1, hkv, g * n, m), v.permute(0, 2, 1, 3))
        o = torch.where(tot > 0, o.view(-1, hkv, g, n, D) / tot, 0.0)
        to = rows[there]
        out[to] = o.permute(0, 3, 1, 2, 4).reshape(-1, n, hq, D)[there]
        lse[to] = (mx + tot.log())[..., 0].permute(0, 3, 1, 2).reshape(-1, n, hq)[there]
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_read(s):
    page, slots = s["case"]["page"], s["slots"]
    at = slots.clamp_min(0)
    at = (at // page, at % page)
    there = (slots >= 0)[:, None, None]
    got = {}
    for x in ("k", "v"):
        y = torch.where(there, _values(_take(s[x], at), s[x + "e"][at]), 0.0)
        got[x] = y.to(_dtype(s["case"]))
    return got


def _plain_store(s):
    page, slots = s["case"]["page"], s["slots"]
    new = slots >= 0
    to = slots[new]
    to = (to // page, to % page)
    for x in ("k", "v"):
        c, b = _quantised(s[x + "_new"].float(), s["case"]["fmt"])
        s[x].view(torch.uint8)[to], s[x + "e"][to] = c.view(torch.uint8)[new], b[new]
    return {**_plain_read(s), "k_exps": s["ke"], "v_exps": s["ve"]}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"attend": _plain_attend, "store": _plain_store, "read": _plain_read}[kind](state)
    L, s = _lib(), state
    cache = (s["k"], s["ke"], s["v"], s["ve"])
    if kind == "attend":
        out, lse = L.pair_attend_paged_q8(s["q"], *cache, s["table"], s["kv"], s["cu"],
                                          scale=s["scale"], max_new=s["case"]["n_hi"],
                                          out=s["out"], lse=s["lse"], ws=s["ws"],
                                          dev_err=s["err"])
        return {"out": out, "lse": lse}
    if kind == "store":
        L.pair_cache_append_q8(s["k_new"], s["v_new"], s["slots"], *cache, dev_err=s["err"])
    k, v = L.pair_cache_read_q8(s["slots"], *cache, k=s["k_out"], v=s["v_out"], dev_err=s["err"])
    return {"k": k, "v": v, **({"k_exps": s["ke"], "v_exps": s["ve"]} if kind == "store" else {})}


# ------------------------------------------------------------------ the work
def work(case):
    """Expected over the seeds, where lengths are drawn."""
    size = 2 if case["dtype"] == "bf16" else 4
    per_token = 2 * case["hkv"] * (case["D"] + 1)  # codes and exponents of keys and values
    if case["kind"] == "attend":
        R = case["B"] * case["G"]
        n = (case["n_lo"] + case["n_hi"]) / 2
        if case["dist"] == "lognormal":
            x = np.exp(math.log(case["ctx_lo"]) +
                       0.9 * np.random.default_rng(0).standard_normal(20000))
            ctx = float(np.clip(x, case["prompt"], case["ctx_hi"]).mean())
        else:
            lo, hi, least = case["ctx_lo"], case["ctx_hi"], case["prompt"]
            ctx = float(np.maximum(np.linspace(lo, hi, 1001), least).mean())
        tokens = R * (ctx + n) - (R - case["B"]) * case["prompt"]  # a shared prompt is read once
        rows = R * n * case["hq"]
        return {"bytes": tokens * per_token + rows * (2 * case["D"] * size + 4)
                + 4 * R * (ctx + n) / case["page"],
                "flops": 4 * rows * case["D"] * (ctx + (n + 1) / 2)}
    plain = 2 * case["hkv"] * case["D"] * size
    # Stored rows come in once, the stored form is written and the values read
    # back go out; the stored form need not be read from memory again.
    return {"bytes": case["T"] * (8 + per_token + plain * (2 if case["kind"] == "store" else 1)),
            "flops": 0}


# ------------------------------------------------------------------ in 64 bits
def _two_to(e):
    """2^e for whole numbers in 64 bits, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_values(codes, b):
    return codes.double() * _two_to(b.long() - 127)[..., None]


def _exact_attend(s):
    case = s["case"]
    page, g = case["page"], case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    for i, m in enumerate(s["kv_host"]):
        a, b = s["cu_host"][i], s["cu_host"][i + 1]
        pos = torch.arange(m, device=DEV)
        where = s["table"][i].long()[pos // page]
        for h in range(case["hkv"]):
            at = (where, pos % page, h)
            k = _exact_values(_take(s["k"], at), s["ke"][at])
            v = _exact_values(_take(s["v"], at), s["ve"][at])
            for j in range(a, b, 512):
                e = min(b, j + 512)
                x = torch.einsum("thd,kd->thk", s["q"][j:e, h * g:(h + 1) * g].double(), k)
                x = x * s["scale"]
                limit = m - (b - torch.arange(j, e, device=DEV))  # the last key that a row sees
                x = torch.where(pos[None, None] > limit[:, None, None], -math.inf, x)
                z = torch.logsumexp(x, -1) if m else torch.full(x.shape[:2], -math.inf,
                                                               dtype=torch.float64, device=DEV)
                w = torch.where(z[..., None] == -math.inf, 0.0, torch.exp(x - z[..., None]))
                out[j:e, h * g:(h + 1) * g] = torch.einsum("thk,kd->thd", w, v)
                lse[j:e, h * g:(h + 1) * g] = z
    return {"out": out, "lse": lse}


def _exact_stored(x, fmt):
    """The values that rows x stand for once they are stored, by the definition:
    the least exponent is looked for from below."""
    x = x.double()
    most, round_at = (127.0, 127.5) if fmt == "i8" else (448.0, 464.0)
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -127.0)
    for k in range(-126, 122):
        e = torch.where(top * 2.0 ** (1 - k) >= round_at, float(k), e)
    y = x * _two_to(-e)
    if fmt == "i8":
        step = torch.ones_like(y)
    else:  # four significant bits down to 2^-6, then steps of 2^-9
        step = _two_to(torch.frexp(y.abs().clamp_min(2.0 ** -6))[1] - 4)
    q = torch.round(y / step) * step
    assert float(q.abs().max()) <= most
    return q * _two_to(e)


def _exact_rows(s):
    case, page = s["case"], s["case"]["page"]
    got = {}
    for x in ("k", "v"):
        if case["kind"] == "store":
            y = _exact_stored(s[x + "_new"], case["fmt"])
        else:
            at = s["slots"].clamp_min(0)
            at = (at // page, at % page)
            y = _exact_values(_take(s[x], at), s[x + "e"][at])
        got[x] = torch.where((s["slots"] >= 0)[:, None, None], y, 0.0)
    if case["kind"] == "store":
        got.update(k_exps=None, v_exps=None)  # whole numbers
    return got


def exact(case, seed):
    if case["kind"] == "attend" and work(case)["flops"] > 2e12:
        return None
    return (_exact_attend if case["kind"] == "attend" else _exact_rows)(prepare(case, seed))
