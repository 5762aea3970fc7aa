"""The cache in pages, in fp64 and plain integers: page tables and slots of a step, rows into their slots, and
attention of packed rows of new tokens over pages or over the pack itself."""
from __future__ import annotations

import numpy as np


def page_plan(q_len, kv_len, held, table, free, n_free, P, T):
    """The step's tables.  table and free are not changed; returns dict(table, free, cu_q, slots, positions, new_kv_len,
    new_held, new_n_free)."""
    table, stack = np.array(table), list(free)
    B, width = table.shape
    cap, n = len(stack), int(np.clip(n_free, 0, len(stack)))
    held = [int(np.clip(h, 0, width)) for h in held]
    kv_len = [max(0, int(x)) for x in kv_len]
    for b in range(B):
        if q_len[b] < 0:
            for j in range(held[b]):
                if n < cap:
                    stack[n] = table[b, j]
                    n += 1
    there, asked = n, 0
    cu, slots, pos, new_kv, new_held = [0], [-1] * T, [0] * T, [], []
    for b in range(B):
        m = min(max(0, int(q_len[b])), T - cu[-1])
        cu.append(cu[-1] + m)
        if q_len[b] < 0:
            new_kv.append(0)
            new_held.append(0)
            continue
        pages = -(-(kv_len[b] + m) // P)
        fits = pages <= width and kv_len[b] + m < 2 ** 31
        need = max(0, pages - held[b]) if fits and m > 0 else 0
        asked += need
        ok = fits and (need == 0 or asked <= there)
        for j in range(need if ok else 0):
            n -= 1
            table[b, held[b] + j] = stack[n]
        for i in range(m):
            t = kv_len[b] + i
            pos[cu[b] + i] = min(t, 2 ** 31 - 1)
            if ok:
                s = int(table[b, t // P]) * P + t % P
                slots[cu[b] + i] = s if 0 <= s < 2 ** 31 else -1
        new_kv.append(kv_len[b] + (m if ok else 0))
        new_held.append(held[b] + (need if ok else 0))
    return dict(table=table, free=np.array(stack), cu_q=np.array(cu), slots=np.array(slots, dtype=np.int64),
                positions=np.array(pos, dtype=np.int64), new_kv_len=np.array(new_kv), new_held=np.array(new_held),
                new_n_free=n)


def append(pool, new, slots):
    """pool [n_pages, H, P, D] with rows new [T, H, D] at their slots."""
    pool = np.array(pool)
    n, _, P, _ = pool.shape
    for i, s in enumerate(slots):
        if 0 <= s < n * P:
            pool[s // P, :, s % P] = new[i]
    return pool


def gather(pool, row, kv, h):
    """Keys (or values) [kv, D] of a request's pages, cached head h; page numbers outside the pool as the nearest inside."""
    n, _, P, _ = pool.shape
    t = np.arange(kv)
    return pool[np.clip(np.asarray(row)[t // P], 0, n - 1), h, t % P]


def attend(q, K, V, sees, scale):
    """(out [m, D], its weighted mean of |V|, the largest sum of |q k| scale) of rows q [m, D] over keys K and values V [kv, D],
    row i seeing the first sees[i].  What a row does not see has no part in it; a score that is NaN or +inf makes it NaN, one
    of -inf has no weight, a value that is not finite decides its column."""
    q, K, V = (np.asarray(x, dtype=np.float64) for x in (q, K, V))
    out, mean, top = np.zeros(q.shape), np.zeros(q.shape), np.zeros(len(q))
    for i, n in enumerate(sees):
        if n <= 0:
            continue
        with np.errstate(all="ignore"):
            s = (K[:n] @ q[i]) * scale
        if np.isnan(s).any() or np.isposinf(s).any() or np.isneginf(s).all():
            out[i] = np.nan
            continue
        w = np.exp(s - s.max())
        keep = ~np.isneginf(s)
        w, v = w[keep], V[:n][keep]
        fin = np.isfinite(v)
        out[i] = w @ np.where(fin, v, 0) / w.sum()
        mean[i] = w @ np.abs(np.where(fin, v, 0)) / w.sum()
        odd = ~fin.all(0)
        with np.errstate(all="ignore"):
            out[i, odd] = np.where(fin, 0, v).sum(0)[odd]
        top[i] = (np.abs(K[:n][keep]) @ np.abs(q[i])).max() * scale
    return out, mean, top
