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


# ------------------------------------------------------------------ normalised heads

def norm_rotate(x, g, eps, pos=None, cos=None, sin=None):
    """fp16 [T, H, D] divided by each head's root mean square, times g ([D] or [H, D]; None: as it is), and rotated as in
    rotate() if there are tables: float64, rounded once"""
    y = x.astype(np.float64)
    if g is not None:
        with np.errstate(invalid="ignore", divide="ignore"):
            y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * g.astype(np.float64)
    if cos is not None:
        p = np.clip(pos, 0, cos.shape[0] - 1)
        c, s = cos[p][:, None, :].astype(np.float64), sin[p][:, None, :].astype(np.float64)
        lo, hi = np.split(y, 2, -1)
        y = np.concatenate([lo * c - hi * s, hi * c + lo * s], -1)
    with np.errstate(over="ignore"):
        return y.astype(np.float16)


# ------------------------------------------------------------------ shared pages, forks, compactions

def _give_back(shared, ring, head, count, took):
    back = [p for p in range(len(shared)) if shared[p] < 0]
    for i, p in enumerate(back):
        ring[(head + count + i) % len(ring)] = p
        shared[p] = 0
    return [(head + took) % len(ring), count - took + len(back)]


def kv_fork(kv_len, parent, page, table, shared, ring, state, table_out):
    """(kv_len, table, shared, copy_src, copy_dst, ring, state, status) after the requests went on as copies of others"""
    kv_len, parent, table, ring = [int(x) for x in kv_len], [int(x) for x in parent], np.array(table), np.array(ring)
    shared, out = np.maximum(np.array(shared), 0), np.array(table_out)
    B, (head, count), n_pages = len(kv_len), (int(x) for x in state), len(ring)
    up = lambda n: -(-n // page)
    cap = table.shape[1] * page
    wrong = not (0 <= head < n_pages and 0 <= count <= n_pages) or any(p < -1 or p >= B for p in parent) or any(n < 0 or n > cap for n in kv_len)

    def refused(status):
        for b in range(B):
            n = min(up(max(kv_len[b], 0)), table.shape[1])
            out[b, :n] = table[b, :n]
        return kv_len, out, shared, [-1] * B, [-1] * B, ring, [head, count], status
    if wrong:
        return refused(-1)
    there = lambda p: 0 <= p < n_pages
    joint = lambda b: there(table[b, up(kv_len[b]) - 1]) and shared[table[b, up(kv_len[b]) - 1]] > 0
    copies, first = [], set()
    for b, p in enumerate(parent):
        if p >= 0 and kv_len[p] % page and (p in first or joint(p)):
            copies.append(b)
        first.add(p)
    if len(copies) > count:
        return refused(len(copies) - count)
    src, dst, holders = [-1] * B, [-1] * B, np.zeros(n_pages, dtype=np.int64)
    for b in range(B):
        for p in table[b, :up(kv_len[b])]:
            if there(p):
                holders[p] -= 1
    for b, p in enumerate(parent):
        if p < 0:
            continue
        n = up(kv_len[p])
        out[b, :n] = table[p, :n]
        if b in copies:
            src[b], dst[b] = int(table[p, n - 1]), int(ring[(head + copies.index(b)) % n_pages])
            out[b, n - 1] = dst[b]
        for q in table[p, :n - 1 if b in copies else n]:
            if there(q):
                holders[q] += 1
    if count + (shared + holders < 0).sum() > n_pages:
        return refused(-1)
    shared = shared + holders
    state = _give_back(shared, ring, head, count, len(copies))
    return [kv_len[p] if p >= 0 else 0 for p in parent], out, shared, src, dst, ring, state, 0


def kv_compact(kv_len, stay, cu, keep, page, table, shared, ring, state, table_out):
    """(kv_len, table, shared, ring, state, status, moves) after the requests lost tokens; moves: (new page, the tokens that it
    gets as (page, slot) pairs)"""
    kv_len, stay, cu, keep = ([int(x) for x in a] for a in (kv_len, stay, cu, keep))
    table, ring, shared, out = np.array(table), np.array(ring), np.maximum(np.array(shared), 0), np.array(table_out)
    B, (head, count), n_pages, cap = len(kv_len), (int(x) for x in state), len(ring), table.shape[1] * page
    up = lambda n: -(-n // page)

    def refused(status):
        for b in range(B):
            n = min(up(max(kv_len[b], 0)), table.shape[1])
            out[b, :n] = table[b, :n]
        return kv_len, out, shared, ring, [head, count], status, []
    wrong = not (0 <= head < n_pages and 0 <= count <= n_pages) or any(n < 0 or n > cap for n in kv_len) or any(s < 0 for s in stay)
    wrong = wrong or any(not 0 <= a <= b <= len(keep) for a, b in zip(cu, cu[1:]))
    if not wrong:
        for b in range(B):
            mine = keep[cu[b]:cu[b + 1]]
            wrong = wrong or any(x < stay[b] or x >= kv_len[b] for x in mine) or any(x >= y for x, y in zip(mine, mine[1:]))
    if wrong:
        return refused(-1)
    plan, need = [], 0
    for b in range(B):
        tokens = list(range(min(stay[b], kv_len[b]))) + keep[cu[b]:cu[b + 1]]
        n, some = len(tokens), cu[b + 1] > cu[b]
        same = stay[b] // page if some else up(n)
        if not some and n < kv_len[b] and n % page:
            last = table[b, up(n) - 1]
            same -= bool(0 <= last < n_pages and shared[last] > 0)
        plan.append((tokens, same))
        need += up(n) - same
    if need > count:
        return refused(need - count)
    took, moves, held = 0, [], np.zeros(n_pages, dtype=np.int64)
    for b, (tokens, same) in enumerate(plan):
        out[b, :same] = table[b, :same]
        for j in range(same, up(len(tokens))):
            new = int(ring[(head + took) % n_pages])
            out[b, j] = new
            took += 1
            moves.append((new, [(int(table[b, i // page]), i % page) for i in tokens[j * page:(j + 1) * page]]))
        for p in table[b, same:up(kv_len[b])]:
            if 0 <= p < n_pages:
                held[p] -= 1
    if count + (shared + held < 0).sum() > n_pages:
        return refused(-1)
    shared = shared + held
    state = _give_back(shared, ring, head, count, took)
    return [len(t) for t, _ in plan], out, shared, ring, state, 0, moves


def kv_move(codes, exps, moves, transposed):
    """the codes and exponents of one layer (keys, or values: transposed) after kv_compact's moves; new arrays"""
    old = codes.transpose(0, 1, 3, 2) if transposed else codes
    codes, new_exps = codes.copy(), exps.copy()
    view = codes.transpose(0, 1, 3, 2) if transposed else codes
    for to, tokens in moves:
        for h in range(old.shape[1]):
            e = max(int(exps[p, h]) for p, _ in tokens)
            view[to, h] = 0
            for i, (p, slot) in enumerate(tokens):
                view[to, h, i] = np.rint(old[p, h, slot].astype(np.float64) * 2.0 ** (int(exps[p, h]) - e))
            new_exps[to, h] = e
    return codes, new_exps


# ------------------------------------------------------------------ log probabilities

def logprobs(x, tokens, n_top, scale=1.0):
    """Rows of logits x [T, V] (fp16 or float32): dict of logprob, entropy, top_idx, top_logprob in float64, and of bounds on
    what float32 arithmetic may be off, in units of d = 2^-24, to first order:
      z = (x - m) c, c = scale log2(e): a difference, a product, c's two roundings: 4 d |z|
      2^z: ln 2 times that, and the exponential's own 2 d, relative
      S, E: sums of a few terms in 10 steps, the others in float64; z is relative to a logit less than a factor of two below the
      largest, 1 more than |z|, and is brought to a larger one by a rounded factor (2 d) for every power of two or more, 3 d |z| + 2 d;
      lanes, wavefronts and pieces are joined by a factor each, 10 d: 24 d and 3 d |z|
      log2 S: 2 d of itself, and S's relative error over ln 2; differences, products and factors: d or two of the result"""
    T, V = x.shape
    d, steps = 2.0 ** -24, 24
    r = dict(logprob=np.full(T, np.nan), entropy=np.full(T, np.nan), top_idx=np.full((T, n_top), -1, dtype=np.int64),
             top_logprob=np.full((T, n_top), np.nan), logprob_bound=np.zeros(T), entropy_bound=np.zeros(T), top_bound=np.zeros((T, n_top)))
    for t in range(T):
        y = x[t].astype(np.float64)
        if np.isnan(y).any() or y.max() == np.inf or y.max() == -np.inf:
            continue
        with np.errstate(invalid="ignore"):
            z = (y - y.max()) * float(scale)
            w = np.exp(z)
            lse = np.log1p(w.sum() - 1.0) if w.sum() < 1.5 else np.log(w.sum())
            p = w / w.sum()
            lp = z - lse
            size = np.where(p > 0, p * np.abs(z), 0.0).sum()
            square = np.where(p > 0, p * z * z, 0.0).sum()
        S = 7 * size + 2 + steps                                                        # relative error of S over d
        log_err = S + 2 * abs(lse)
        at = lambda v: d * (4 * np.abs(v) + log_err + 4 * np.abs(v - lse)) + 2.0 ** -149
        r["entropy"][t] = -(p[p > 0] * lp[p > 0]).sum()
        r["entropy_bound"][t] = d * (log_err + 7 * (square + 2 * size + 1) + (steps + 8 + S) * (size + 1) + 4 * (abs(lse) + size))
        tok = -1 if tokens is None else int(tokens[t])
        if 0 <= tok < V:
            r["logprob"][t] = lp[tok]
            r["logprob_bound"][t] = 0 if np.isinf(z[tok]) else at(z[tok])
        last = np.partition(-y, n_top - 1)[n_top - 1] if n_top else -np.inf
        among = np.flatnonzero(-y <= last) if n_top else np.zeros(0, dtype=np.int64)
        order = among[np.argsort(-(y[among] + 0.0), kind="stable")][:n_top]
        r["top_idx"][t], r["top_logprob"][t] = order, lp[order]
        fin = np.isfinite(z[order])
        r["top_bound"][t, fin] = at(z[order][fin])
    return r
