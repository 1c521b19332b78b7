"""Plain definitions of the serving calls in float64 and whole numbers (numpy): the page map of a step, the write into the
8-bit cache, and attention with the bound on its rounding errors."""
from __future__ import annotations

import numpy as np

E_ZERO = -30


def kv_map(kv_len, n_new, table, page, ring, state, T):
    """(kv_len, cu_new, pos, slot, table, ring, state, status) after one step; one request, token and page at a time."""
    kv_len, n_new = [int(x) for x in kv_len], [int(x) for x in n_new]
    table, ring = np.array(table), np.array(ring)
    B, (head, count), n_pages = len(kv_len), (int(x) for x in state), len(ring)
    up = lambda n: -(-n // page)
    refused = (kv_len, [0] * (B + 1), [0] * T, [-1] * T, table.copy(), ring.copy(), [head, count])
    wrong = not (0 <= head < n_pages and 0 <= count <= n_pages)
    need = back = tokens = 0
    for past, add in zip(kv_len, n_new):
        after = past + max(add, 0)
        if past < 0 or add < -1 or after > table.shape[1] * page:
            wrong = True
            continue
        tokens += max(add, 0)
        need += up(after) - up(past) if add > 0 else 0
        back += up(past) if add < 0 else 0
    if wrong or tokens > T or count + back > n_pages:
        return refused + (-1,)
    if need > count:
        return refused + (need - count,)
    old_ring, old_table = ring.copy(), table.copy()
    took = gave = 0
    lens, cu, pos, slot = [], [0], [], []
    for b, (past, add) in enumerate(zip(kv_len, n_new)):
        if add < 0:
            for j in range(up(past)):
                ring[(head + count + gave) % n_pages] = old_table[b, j]
                gave += 1
        for p in range(past, past + max(add, 0)):
            if p % page == 0:
                table[b, p // page] = old_ring[(head + took) % n_pages]
                took += 1
            pos.append(p)
            at = int(table[b, p // page])
            slot.append(at * page + p % page if 0 <= at < n_pages else -1)
        lens.append(0 if add < 0 else past + add)
        cu.append(len(pos))
    rest = T - len(pos)
    return lens, cu, pos + [0] * rest, slot + [-1] * rest, table, ring, [(head + took) % n_pages, count - took + gave], 0


def rotate(x, pos, cos, sin):
    """fp16 [T, H, D]: pairs (i, i + D/2) turned by the angle of (pos, i), float64, rounded once"""
    p = np.clip(pos, 0, cos.shape[0] - 1)
    c, s = cos[p][:, None, :].astype(np.float64), sin[p][:, None, :].astype(np.float64)
    half = x.shape[-1] // 2
    lo, hi = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1).astype(np.float16)


def exponent(top):
    """the smallest e with top <= 127 * 2^e; infinities count as 2^16, zero as E_ZERO"""
    top = min(float(top), 65536.0)
    e = E_ZERO
    while top > 127.0 * 2.0 ** e:
        e += 1
    return e


def kv_append(x, slot, codes, exps, transposed):
    """fp16 [T, H, D] into codes [n_pages, H, page, D] (or [n_pages, H, D, page]) and exps [n_pages, H]; new arrays"""
    codes, exps = codes.copy(), exps.copy()
    view = codes.transpose(0, 1, 3, 2) if transposed else codes
    n_pages, H, page, _ = view.shape
    t = 0
    while t < len(slot):
        if not 0 <= slot[t] < n_pages * page:
            t += 1
            continue
        p, off, n = slot[t] // page, slot[t] % page, 1
        while t + n < len(slot) and slot[t + n] == slot[t] + n and off + n < page:
            n += 1
        for h in range(H):
            rows = x[t:t + n, h].astype(np.float64)
            e = exponent(np.abs(rows).max())
            if off:
                had = int(exps[p, h])
                e = max(e, had)
                view[p, h, :off] = np.rint(view[p, h, :off].astype(np.float64) * 2.0 ** (had - e))
            view[p, h, off:off + n] = np.clip(np.rint(rows * 2.0 ** -e), -128, 127)
            exps[p, h] = e
        t += n
    return codes, exps


def cache_rows(codes, exps, table, L, h, transposed):
    """the L x D values of key head h that a request's table row stands for"""
    n_pages = codes.shape[0]
    page = codes.shape[3 if transposed else 2]
    rows, there = [], []
    for j in range(-(-L // page)):
        p = int(table[j])
        ok = 0 <= p < n_pages
        c = codes[p if ok else 0, h].astype(np.float64) * 2.0 ** int(exps[p if ok else 0, h])
        rows.append(c.T if transposed else c)
        there += [ok] * page
    D = codes.shape[2 if transposed else 3]
    return (np.concatenate(rows)[:L] if rows else np.zeros((0, D))), np.array(there[:L], dtype=bool)


def attention(q, k, v, past, causal=True, scale=None, there=None, offset=None):
    """q [n, D], k and v [m, D], float64: (o [n, D], bound [n, D]).  Query i sees keys j <= past + i (past = m - n) if causal, and
    only those that are there.  offset [n]: added to X below, for keys that are multiplied in a form with larger products.
    bound: how far a result with the roundings that include/agq.h allows can be from o:
      scores: fp32 sums of D exact products, then a multiply-add and a difference; relative to the sum of the products'
              magnitudes X (in units of the exponent of 2) D + 4 roundings of 2^-24, twice (its own and the maximum's), which
              the exponential turns into a relative error of the weight of ln 2 times that; the exponential itself 2^-22
      weights: fp16 in the second product, 2^-11 of each; below 2^-24 of the largest, half of fp16's smallest step instead,
              2^-25 over the factor of at least 2^10 that they are raised by
      sums: fp32, m terms of the softmax's and of the product's
      result: one rounding to fp16, 2^-11 of it or 2^-25, and a quotient's."""
    n, D = q.shape
    m = k.shape[0]
    scale = D ** -0.5 if scale is None else scale
    o, bound = np.zeros((n, D)), np.zeros((n, D))
    for i in range(n):
        see = np.ones(m, dtype=bool) if there is None else there.copy()
        if causal:
            see[max(0, past + i + 1):] = False
        if not see.any():
            continue
        kk, vv = k[see], v[see]
        with np.errstate(invalid="ignore", over="ignore"):
            s = kk @ q[i] * scale
            w = np.exp(s - s.max())
            total = w.sum()
            o[i] = (w @ vv) / total
            X = ((np.abs(kk) @ np.abs(q[i])).max() + (0.0 if offset is None else offset[i])) * scale * np.log2(np.e)
            A = (w @ np.abs(vv)) / total
            rel = 2 * np.log(2) * (D + 4) * 2.0 ** -24 * X + 2.0 ** -22
            bound[i] = (2.0 ** -11 + 2 * rel + 2 * (len(kk) + 64) * 2.0 ** -24) * A + len(kk) * 2.0 ** -35 * np.abs(vv).max(0) / total \
                + 2.0 ** -11 * np.abs(o[i]) + 2.0 ** -25
    return o, bound
