"""64-bit numpy forms of the rollout step's operators: pages and slots,
attention over a paged cache, verification of drafted tokens. Loops over
requests and rows, from the definitions."""
import math

import numpy as np


def pages_extend(lens, held, n_new, free_pages, free_count, table, page, T):
    """Returns dict(table, kv_len, held, cu, slots, taken, error)."""
    R, width = table.shape
    table = table.copy()
    old = table.copy()
    avail = min(max(int(free_count), 0), len(free_pages))
    kv_len, held_out = np.zeros(R, np.int64), np.zeros(R, np.int64)
    cu, slots = np.zeros(R + 1, np.int64), np.full(T, -1, np.int64)
    row, used, taken, error = 0, 0, 0, False
    for i in range(R):
        n = max(int(n_new[i]), 0)
        total = -(-(int(lens[i]) + n) // page)
        bad = (lens[i] < 0 or held[i] < 0 or n_new[i] < 0 or held[i] > width
               or held[i] * page < lens[i] or total > width)
        need = 0 if bad else max(total - int(held[i]), 0)
        ok = not bad and (need == 0 or used + need <= avail) and row + n <= T
        error |= not ok
        kv_len[i] = lens[i] + n if ok else max(int(lens[i]), 0)
        held_out[i] = held[i] + (need if ok else 0)
        if ok:
            for j in range(need):
                table[i, held[i] + j] = free_pages[used + j]
            if need:
                taken = max(taken, used + need)
            for j in range(n):
                pos = int(lens[i]) + j
                at = pos // page
                pg = int(old[i, at]) if at < held[i] else int(table[i, at])
                slots[row + j] = pg * page + pos % page
        row += n
        used += need
        cu[i + 1] = min(row, T)
    return dict(table=table, kv_len=kv_len, held=held_out, cu=cu, slots=slots, taken=taken,
                error=error)


def attend_paged(q, k_cache, v_cache, table, kv_len, cu, scale):
    """q [T, Hq, D], caches [pages, page, Hkv, D] in fp64. Returns out, lse,
    and per row and head the sizes that error bounds need: mag [T, Hq, D] =
    sum_k p_k |v_k| and size [T, Hq] = max_k scale sum_d |q_d k_d|."""
    T, Hq, D = q.shape
    page, Hkv = k_cache.shape[1:3]
    g = Hq // Hkv
    out, mag = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, size = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    for i in range(len(kv_len)):
        n, m = int(cu[i + 1] - cu[i]), int(kv_len[i])
        if n == 0 or m == 0:
            continue
        pos = np.arange(m)
        pg = np.asarray(table[i])[pos // page]
        for j in range(n):
            see = min(max(m - n + j + 1, 0), m)
            if see == 0:
                continue
            t = int(cu[i]) + j
            for h in range(Hkv):
                k = k_cache[pg[:see], pos[:see] % page, h]
                v = v_cache[pg[:see], pos[:see] % page, h]
                for hh in range(h * g, (h + 1) * g):
                    s = scale * (k @ q[t, hh])
                    z = s.max()
                    w = np.exp(s - z)
                    lse[t, hh] = z + math.log(w.sum())
                    w /= w.sum()
                    out[t, hh] = w @ v
                    mag[t, hh] = w @ np.abs(v)
                    size[t, hh] = abs(scale) * (np.abs(k) @ np.abs(q[t, hh])).max()
    return out, lse, mag, size


def verify_drafts(p, ids, cu, u, u_draw, q=None):
    """p, q [T, V] float32 (rows widened from their type). The acceptance and
    the weights are the definition's fp32 product and difference; their sums
    are Python integers. Returns dict(ids, logp, n, error bits)."""
    T, V = p.shape
    R = len(cu) - 1
    out, logp, n_emit = np.full(T, -1, np.int64), np.zeros(T), np.zeros(R, np.int64)
    bad_id = bad_p = False

    def draw(x, t):
        w = [int(math.floor(min(max(float(v), 0.0), 1.0) * 2.0 ** 40)) if v == v else 0 for v in x]
        total = sum(w)
        if total == 0:
            return None
        at = max(min(int(float(t) * float(total)), total - 1), 0)
        c = 0
        for v in range(V):
            c += w[v]
            if c > at:
                return v
        raise AssertionError

    for i in range(R):
        lo, hi = int(cu[i]), int(cu[i + 1])
        for t in range(lo, hi):
            drafted, src = t + 1 < hi, p[t]
            if drafted:
                y = int(ids[t + 1])
                if 0 <= y < V:
                    qy = np.float32(1.0) if q is None else q[t, y]
                    if np.float32(u[t]) * qy < p[t, y]:
                        out[t], logp[t] = y, math.log(float(p[t, y]))
                        n_emit[i] += 1
                        continue
                    if q is None:
                        src = p[t].copy()
                        src[y] = 0.0
                else:
                    bad_id = True
                if q is not None:
                    src = p[t] - q[t]
            tok = draw(src, u_draw[i])
            if tok is None:
                tok = draw(p[t], u_draw[i])
            if tok is None:
                bad_p = True
            else:
                out[t], logp[t] = tok, math.log(float(p[t, tok]))
                n_emit[i] += 1
            break
    return dict(ids=out, logp=logp, n=n_emit, bad_id=bad_id, bad_p=bad_p)


def store_q8(x, fmt):
    """Rows x [.., D] as they are held in 8 bits: (codes, exponent bytes), the
    codes as the numbers they are ("i8" whole numbers, "e4m3" values of that
    type). The exponent is looked for from below, one at a time."""
    x = np.asarray(x, np.float64)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(top)
    limit = 127.5 if fmt == "i8" else 464.0  # what is below rounds to 127, to 448
    b = np.zeros(top.shape, np.int64)
    for _ in range(255):
        b += (b < 254) & (np.where(bad, 0.0, top) * 2.0 ** (127 - b) >= limit)
    y = np.where(bad[..., None], 0.0, x) * 2.0 ** (127 - b)[..., None]
    if fmt == "i8":
        c = np.rint(y)
    else:  # four significant bits down to 2^-6, steps of 2^-9 below
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -6))) - 3)
        c = np.rint(y / step) * step
    return c, np.where(bad, 255, b)


def values_q8(codes, exps):
    """What codes and exponent bytes stand for."""
    s = np.where(np.asarray(exps) == 255, np.nan, 2.0 ** (np.asarray(exps, np.float64) - 127))
    return np.asarray(codes, np.float64) * s[..., None]
