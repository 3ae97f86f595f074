"""Operators of the rollout continuation step, as timed cases.

A rollout that the allocation step continues is generated with drafted tokens:
every step the continued requests get cache pages for their chunk of new
tokens (pair_pages_extend), the chunk's keys and values go into those pages
(pair_cache_append), its queries attend over the paged cache
(pair_attend_paged), and the drafted tokens are verified against the target's
probabilities (pair_verify_drafts), which also gives the log-probabilities
that the clipped surrogate takes as the old ones.

The plain forms are elementary torch operations in 32 bits, request by request
where the lengths differ; a scheduler's host copy of the lengths is part of
the state. `exact` computes the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
FIXED = float(2 ** 40)  # sampling weights are integers in units of 2^-40


# ---------------------------------------------------------------- the cases
def listed():
    return [
        # One rollout generating token by token: 16 query and 8 key heads of
        # 128 over a few hundred cached tokens. Latency is all there is.
        dict(name="attend_1x1", kind="attend", dtype="bf16", B=1, G=1, hq=16, hkv=8, D=128, page=16,
             prompt=0, dist="uniform", ctx_lo=700, ctx_hi=700, n_lo=1, n_hi=1, layout="token"),
        # 8 prompts x 8 rollouts of 256 to 2048 tokens, a token each.
        dict(name="attend_8x8_token", kind="attend", dtype="bf16", B=8, G=8, hq=16, hkv=8, D=128,
             page=16, prompt=192, dist="uniform", ctx_lo=256, ctx_hi=2048, n_lo=1, n_hi=1,
             layout="head"),
        # 16 x 16 rollouts of 512 to 4096 tokens on 32/8 heads, each with
        # four drafted tokens behind its last one.
        dict(name="attend_16x16_drafts", kind="attend", dtype="bf16", B=16, G=16, hq=32, hkv=8,
             D=128, page=32, prompt=512, dist="uniform", ctx_lo=512, ctx_hi=4096, n_lo=5, n_hi=5,
             layout="token"),
        # The heavy-tailed workload: 32 x 16 rollouts, median 1500 tokens,
        # capped at 16384, a token each: the most bytes one call reads.
        dict(name="attend_32x16_skew", kind="attend", dtype="bf16", B=32, G=16, hq=16, hkv=8, D=128,
             page=64, prompt=256, dist="lognormal", ctx_lo=1500, ctx_hi=16384, n_lo=1, n_hi=1,
             layout="token"),
        # Chunks of prompts and of continued prefixes scored at once: ragged
        # chunks of up to 2048 tokens behind up to 6144 cached ones.
        dict(name="attend_chunks_4", kind="attend", dtype="bf16", B=4, G=1, hq=32, hkv=8, D=128,
             page=16, prompt=0, dist="uniform", ctx_lo=1000, ctx_hi=6144, n_lo=1025, n_hi=2048,
             layout="token"),
        # The fp32 reference head's 4 x 8 rollouts, heads of 64, pages of 24.
        dict(name="attend_f32_4x8", kind="attend", dtype="f32", B=4, G=8, hq=4, hkv=2, D=64, page=24,
             prompt=0, dist="uniform", ctx_lo=32, ctx_hi=640, n_lo=3, n_hi=3, layout="token"),
        # Pages of one token each for 8 x 8 rollouts.
        dict(name="pages_8x8", kind="pages", R=64, page=16, ctx_lo=256, ctx_hi=2048, n_lo=1, n_hi=1),
        # Every candidate of 256 groups of 16 admitted at once, with prefixes
        # of up to 256 tokens.
        dict(name="pages_4096", kind="pages", R=4096, page=16, ctx_lo=0, ctx_hi=1024, n_lo=1,
             n_hi=256),
        # New keys and values of 64 tokens, and of four chunks of 2048.
        dict(name="append_64", kind="append", dtype="bf16", T=64, hkv=8, D=128, page=16,
             pages=4096, layout="token"),
        dict(name="append_8192", kind="append", dtype="bf16", T=8192, hkv=8, D=128, page=16,
             pages=4096, layout="head"),
        # Four drafted tokens for one prompt's 4 rollouts and for 16 x 16
        # rollouts, on the 151,936 vocabulary.
        dict(name="verify_4x4", kind="verify", dtype="f32", R=4, K_lo=4, K_hi=4, V=151936, q=True),
        dict(name="verify_256x4", kind="verify", dtype="f32", R=256, K_lo=4, K_hi=4, V=151936,
             q=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "attend", "attend", "pages", "append", "verify",
                       "verify"))
    layout = rng.choice(("token", "head"))
    if kind == "pages":
        n_hi = _log_int(rng, 1, 512)
        R = _log_int(rng, 1, min(4096, max(1, (1 << 19) // n_hi)))
        return dict(kind=kind, R=R, page=rng.choice((1, 8, 16, 24, 32, 64, 128)),
                    ctx_lo=0, ctx_hi=_log_int(rng, 1, 2048), n_lo=rng.choice((0, min(1, n_hi), n_hi)),
                    n_hi=n_hi)
    if kind == "append":
        hkv, D = rng.choice((1, 2, 4, 8)), rng.choice((64, 128))
        return dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "f32")), T=_log_int(rng, 1, 8192),
                    hkv=hkv, D=D, page=rng.choice((8, 16, 24, 64)), pages=2048, layout=layout)
    if kind == "verify":
        V = rng.choice((151936, _log_int(rng, 1000, 151936)))
        K = rng.choice((0, 1, 2, 4, 7))
        R = _log_int(rng, 1, max(1, min(512, 256 * 5 * 151936 // (V * (K + 1)))))
        return dict(kind=kind, dtype=rng.choice(("f32", "f32", "bf16")), R=R,
                    K_lo=rng.choice((0, K)), K_hi=K, V=V, q=rng.random() < 0.7)
    f32 = rng.random() < 0.2
    hq, hkv = rng.choice(((16, 8), (32, 8), (8, 8), (4, 1), (6, 2), (15, 3), (16, 1)))
    c = dict(kind=kind, dtype="f32" if f32 else "bf16", G=rng.choice((1, 4, 8, 16)), hq=hq, hkv=hkv,
             D=rng.choice((64, 128, 128, 128, 256) if not f32 else (64, 128)),
             page=rng.choice((8, 16, 16, 32, 64, 128, 24)))
    n_hi = rng.choice((1, rng.randint(2, 8), _log_int(rng, 9, 2048)))
    n_lo = rng.choice((n_hi, n_hi // 2, 0)) if n_hi > 1 else 1
    skew = rng.random() < 0.25
    ctx_hi = _log_int(rng, 16, 16384 if not f32 else 1024)
    ctx_lo = max(1, ctx_hi // 8) if skew else rng.choice((0, ctx_hi // 2, ctx_hi))
    mean = (ctx_lo * 1.5 if skew else (ctx_lo + ctx_hi) / 2) + n_hi
    most_bytes = 4.0e9 if not f32 else 2.0e8
    most_flops = 3.5e11 if not f32 else 2e10
    size = 4 if f32 else 2
    R = min(512, most_bytes / (2 * size * hkv * c["D"] * mean),
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


def _gen(seed, device=DEV):
    g = torch.Generator(device=device)
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


def _cache(case, g, pages):
    """A filled cache [pages, page, hkv, D], laid out by token or by head."""
    page, hkv, D = case["page"], case["hkv"], case["D"]
    shape = (pages, page, hkv, D) if case["layout"] == "token" else (pages, hkv, page, D)
    x = torch.empty(shape, dtype=_dtype(case), device=DEV)
    x.normal_(generator=g)
    return x if case["layout"] == "token" else x.permute(0, 2, 1, 3)


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
    s = dict(case=case, kv_host=kv.tolist(), cu_host=cu.tolist(), q=q,
             k=_cache(case, g, pages), v=_cache(case, g, pages),
             table=torch.from_numpy(table).to(DEV), kv=torch.from_numpy(kv.astype(np.int32)).to(DEV),
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


def _prepare_pages(case, seed):
    rng = np.random.default_rng(int(seed))
    R, page = case["R"], case["page"]
    lens = _ints(rng, case["ctx_lo"], case["ctx_hi"], R)
    n = _chunks(rng, case["n_lo"], case["n_hi"], R)
    # Some requests hold a page more than their tokens fill: rejected drafts.
    held = -(-lens // page) + (rng.random(R) < 0.2)
    need = np.maximum(-(-(lens + n) // page) - held, 0)
    width = -(-(case["ctx_hi"] + case["n_hi"]) // page) + 2
    pages = int((held + need).sum()) + 8
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((R, width), -1, np.int32)
    at = 0
    for i in range(R):
        table[i, :held[i]] = order[at:at + held[i]]
        at += int(held[i])

    def dev(x, t=np.int32):
        return torch.from_numpy(np.ascontiguousarray(x.astype(t))).to(DEV)

    T = int(n.sum()) + 3  # a captured step has spare rows
    s = dict(case=case, lens=dev(lens), held=dev(held), n=dev(n), free=dev(order[at:]),
             count=dev(np.array([pages - at])), table=dev(table), T=T)
    if own:
        s["kv"], s["held_out"] = torch.empty_like(s["lens"]), torch.empty_like(s["lens"])
        s["cu"] = torch.empty(R + 1, dtype=torch.int32, device=DEV)
        s["slots"] = torch.empty(T, dtype=torch.int64, device=DEV)
        s["taken"] = torch.empty(1, dtype=torch.int32, device=DEV)
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _prepare_append(case, seed):
    g = _gen(seed)
    T, page, pages, dt = case["T"], case["page"], case["pages"], _dtype(case)
    # Chunks of 64 tokens whose pages come in no order; some rows are spare.
    chunk = 64
    rows = -(-chunk // page)
    n_chunks = -(-T // chunk)
    order = torch.randperm(pages, generator=g, device=DEV)[:n_chunks * rows].view(n_chunks, rows)
    t = torch.arange(T, device=DEV)
    pos = t % chunk
    slots = order[t // chunk, pos // page] * page + pos % page
    slots = torch.where(torch.rand(T, generator=g, device=DEV) < 0.02, -1, slots)
    # Keys and values as one projection leaves them: rows of both, strided.
    kvp = torch.randn((T, 2, case["hkv"], case["D"]), generator=g, device=DEV).to(dt)
    s = dict(case=case, k_new=kvp[:, 0], v_new=kvp[:, 1], slots=slots.to(torch.int64),
             k=_cache(case, g, pages), v=_cache(case, g, pages))
    if own:
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def _prepare_verify(case, seed):
    rng, g = np.random.default_rng(int(seed)), _gen(seed)
    R, V, dt = case["R"], case["V"], _dtype(case)
    K = _chunks(rng, case["K_lo"] + 1, case["K_hi"] + 1, R) - 1
    cu = np.concatenate([[0], np.cumsum(K + 1)])
    T = int(cu[-1])
    p, q = torch.empty((T, V), dtype=dt, device=DEV), None
    ids = torch.empty(T, dtype=torch.int32, device=DEV)
    if case["q"]:
        q = torch.empty((T, V), dtype=dt, device=DEV)
    for a in range(0, T, 64):  # sharp distributions; the drafter's is the target's with noise
        m = min(64, T - a)
        z = 4.0 * torch.randn((m, V), generator=g, device=DEV)
        p[a:a + m] = torch.softmax(z, -1).to(dt)
        d = torch.softmax(z + 0.7 * torch.randn((m, V), generator=g, device=DEV), -1).to(dt)
        if q is not None:
            q[a:a + m] = d
            ids[a:a + m] = torch.multinomial(d.float(), 1, generator=g)[:, 0].to(torch.int32)
        else:  # drafts looked up, not sampled: the target's likely tokens
            ids[a:a + m] = torch.multinomial(p[a:a + m].float().square() + 1e-30, 1,
                                             generator=g)[:, 0].to(torch.int32)
    # ids[cu + j + 1] is what row cu + j predicts: drawn above row by row, so
    # they move down by one; a chunk's first id is its last accepted token.
    ids = torch.roll(ids, 1).contiguous()
    u = torch.rand(T, generator=g, device=DEV)
    us = torch.rand(R, generator=g, device=DEV)
    s = dict(case=case, p=p, q=q, ids=ids, cu=torch.from_numpy(cu.astype(np.int32)).to(DEV),
             u=u, us=us)
    if own:
        s["out"] = torch.empty(T, dtype=torch.int32, device=DEV)
        s["logp"] = torch.empty(T, dtype=torch.float32, device=DEV)
        s["n"] = torch.empty(R, dtype=torch.int32, device=DEV)
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
    return s


def prepare(case, seed):
    return {"attend": _prepare_attend, "pages": _prepare_pages, "append": _prepare_append,
            "verify": _prepare_verify}[case["kind"]](case, seed)


# ------------------------------------------------------------------ one pass
def _plain_attend(s):
    c = s["case"]
    hq, hkv, D, page = c["hq"], c["hkv"], c["D"], c["page"]
    g = hq // hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float32, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, device=DEV)
    cu, kv = s["cu_host"], s["kv_host"]
    for i in range(len(kv)):
        n, m = cu[i + 1] - cu[i], kv[i]
        if n == 0 or m == 0:
            continue
        rows = s["table"][i, :-(-m // page)].long()
        k = s["k"][rows].reshape(-1, hkv, D)[:m].float()
        v = s["v"][rows].reshape(-1, hkv, D)[:m].float()
        qi = s["q"][cu[i]:cu[i + 1]].float().view(n, hkv, g, D).permute(1, 2, 0, 3)
        sc = torch.matmul(qi.reshape(hkv, g * n, D), k.permute(1, 2, 0)).view(hkv, g, n, m)
        sc = sc * s["scale"]
        seen = torch.arange(m, device=DEV) <= torch.arange(m - n, m, device=DEV)[:, None]
        sc.masked_fill_(~seen, -math.inf)
        mx = sc.amax(-1, keepdim=True)
        sc.sub_(torch.where(mx == -math.inf, 0.0, mx)).exp_()
        tot = sc.sum(-1, keepdim=True)
        o = torch.matmul(sc.view(hkv, g * n, m), v.permute(1, 0, 2)).view(hkv, g, n, D)
        o = torch.where(tot > 0, o / tot, 0.0)
        out[cu[i]:cu[i + 1]] = o.permute(2, 0, 1, 3).reshape(n, hq, D)
        lse[cu[i]:cu[i + 1]] = (mx + tot.log())[..., 0].permute(2, 0, 1).reshape(n, hq)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_pages(s):
    page, T, R = s["case"]["page"], s["T"], s["lens"].numel()
    lens, held, n = s["lens"].long(), s["held"].long(), s["n"].long()
    kv = lens + n
    need = ((kv + page - 1) // page - held).clamp_min(0)
    first = need.cumsum(0) - need
    col = torch.arange(s["table"].shape[1], device=DEV) - held[:, None]
    src = (first[:, None] + col).clamp(0, s["free"].numel() - 1)
    table = torch.where((col >= 0) & (col < need[:, None]), s["free"][src], s["table"])
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), n.cumsum(0)])
    t = torch.arange(T, device=DEV)
    i = (torch.searchsorted(cu, t, right=True) - 1).clamp_max(R - 1)
    pos = lens[i] + t - cu[i]
    there = t < cu[R]
    where = torch.where(there, pos // page, 0)
    slots = torch.where(there, table[i, where].long() * page + pos % page, -1)
    return {"table": table, "kv": kv.int(), "held": (held + need).int(), "cu": cu.int(),
            "slots": slots, "taken": need.sum().view(1).int()}


def _plain_append(s):
    page, slots = s["case"]["page"], s["slots"]
    at = slots >= 0
    to = slots[at]
    s["k"][to // page, to % page] = s["k_new"][at]
    s["v"][to // page, to % page] = s["v_new"][at]
    return {"k": s["k"], "v": s["v"]}


def _plain_verify(s):
    p, q, cu = s["p"], s["q"], s["cu"].long()
    T, R = p.shape[0], cu.numel() - 1
    t = torch.arange(T, device=DEV)
    i = torch.searchsorted(cu, t, right=True) - 1
    last = t == cu[1:][i] - 1
    y = torch.where(last, 0, torch.roll(s["ids"], -1)).long()
    pt = p[t, y].float()
    qt = torch.ones_like(pt) if q is None else q[t, y].float()
    stop = last | ~(s["u"] * qt < pt)
    row = torch.full((R,), T, dtype=torch.int64, device=DEV)
    row = row.scatter_reduce(0, i, torch.where(stop, t, T), "amin")
    pr = p[row].float()
    if q is None:
        off = torch.zeros_like(pr).scatter_(1, y[row][:, None], pr.gather(1, y[row][:, None]))
    else:
        off = q[row].float()
    w = torch.where(last[row][:, None], pr, pr - off).clamp_min(0)
    w = (w * FIXED).long()
    w = torch.where((w.sum(1) == 0)[:, None], (pr * FIXED).long(), w)
    c = w.cumsum(1)
    total = c[:, -1]
    at = (s["us"].double() * total.double()).long().minimum(total - 1)
    tok = (c <= at[:, None]).sum(1)
    out = torch.where(t < row[i], y, torch.where(t == row[i], tok[i], -1))
    logp = torch.where(out >= 0, p[t, out.clamp_min(0)].float().log(), 0.0)
    return {"ids": out.int(), "logp": logp, "n": (row - cu[:-1] + 1).int()}


def run(state):
    kind = state["case"]["kind"]
    if not own:
        return {"attend": _plain_attend, "pages": _plain_pages, "append": _plain_append,
                "verify": _plain_verify}[kind](state)
    L, s = _lib(), state
    if kind == "attend":
        out, lse = L.pair_attend_paged(s["q"], s["k"], s["v"], s["table"], s["kv"], s["cu"],
                                       scale=s["scale"], max_new=s["case"]["n_hi"], out=s["out"],
                                       lse=s["lse"], ws=s["ws"], dev_err=s["err"])
        return {"out": out, "lse": lse}
    if kind == "pages":
        kv, held, cu, slots, taken = L.pair_pages_extend(
            s["lens"], s["held"], s["n"], s["free"], s["count"], s["table"], s["case"]["page"],
            s["T"], kv_len=s["kv"], held_out=s["held_out"], cu_new=s["cu"], slots=s["slots"],
            taken=s["taken"], dev_err=s["err"])
        return {"table": s["table"], "kv": kv, "held": held, "cu": cu, "slots": slots,
                "taken": taken}
    if kind == "append":
        L.pair_cache_append(s["k_new"], s["v_new"], s["slots"], s["k"], s["v"], dev_err=s["err"])
        return {"k": s["k"], "v": s["v"]}
    ids, logp, n = L.pair_verify_drafts(s["p"], s["ids"], s["cu"], s["u"], s["us"], q=s["q"],
                                        out_ids=s["out"], logp=s["logp"], n_emit=s["n"],
                                        dev_err=s["err"])
    return {"ids": ids, "logp": logp, "n": n}


# ------------------------------------------------------------------ the work
def work(case):
    """Expected over the seeds, where lengths are drawn."""
    kind = case["kind"]
    if kind == "attend":
        size, R = 2 if case["dtype"] == "bf16" else 4, case["B"] * case["G"]
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
        return {"bytes": 2 * tokens * case["hkv"] * case["D"] * size
                + rows * (2 * case["D"] * size + 4) + 4 * R * (ctx + n) / case["page"],
                "flops": 4 * rows * case["D"] * (ctx + (n + 1) / 2)}
    if kind == "pages":
        tokens = case["R"] * (case["n_lo"] + case["n_hi"]) / 2
        return {"bytes": 24 * case["R"] + tokens * (8 + 8 / case["page"]), "flops": 0}
    if kind == "append":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["T"] * (8 + 4 * case["hkv"] * case["D"] * size), "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    K = (case["K_lo"] + case["K_hi"]) / 2
    rows = 1 + (0.5 if case["q"] else 0)  # the stopping row of p, and of q where a draft stopped it
    return {"bytes": case["R"] * (rows * case["V"] * size + (K + 1) * 24), "flops": 0}


# ------------------------------------------------------------------ in 64 bits
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
            k = s["k"][where, pos % page, h].double()
            v = s["v"][where, pos % page, h].double()
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


def _exact_verify(s):
    p, q, ids = s["p"], s["q"], s["ids"].cpu().numpy()
    cu, u, us = s["cu"].cpu().numpy(), s["u"].cpu().numpy(), s["us"].cpu().numpy()
    T = p.shape[0]
    out, logp, n = np.full(T, -1, np.int32), np.zeros(T), np.zeros(len(us), np.int32)
    for i in range(len(us)):
        for t in range(cu[i], cu[i + 1]):
            pt = p[t].double().cpu().numpy()
            drafted = t + 1 < cu[i + 1]
            qt = None
            if drafted:
                y = ids[t + 1]
                if q is not None:
                    qt = q[t].double().cpu().numpy()
                else:
                    qt = np.where(np.arange(len(pt)) == y, pt, 0.0)
                if float(u[t]) * (qt[y] if q is not None else 1.0) < pt[y]:
                    out[t], logp[t] = y, math.log(pt[y])
                    continue
            w = np.floor(np.maximum(pt - (qt if drafted else 0.0), 0.0) * FIXED)
            if not w.any():
                w = np.floor(pt * FIXED)
            c = np.cumsum(w)
            y = int(np.searchsorted(c, min(math.floor(float(us[i]) * c[-1]), c[-1] - 1), "right"))
            out[t], logp[t] = y, math.log(pt[y])
            n[i] = t - cu[i] + 1
            break
    return {"ids": out, "logp": logp, "n": n}


def _exact_append(s):
    page = s["case"]["page"]
    k, v = s["k"].double(), s["v"].double()
    for t, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            k[slot // page, slot % page] = s["k_new"][t].double()
            v[slot // page, slot % page] = s["v_new"][t].double()
    return {"k": k, "v": v}


def exact(case, seed):
    if case["kind"] == "pages":  # whole numbers
        return None
    if case["kind"] == "attend" and work(case)["flops"] > 2e12:
        return None
    return {"attend": _exact_attend, "append": _exact_append,
            "verify": _exact_verify}[case["kind"]](prepare(case, seed))
