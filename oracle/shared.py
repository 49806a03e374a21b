"""Plain fp64 statements of the operators on caches whose prefixes requests share: attention with its
log-sum-exp, the weight that tokens get, and eviction by it.  Pools are slot-major here
([..., n_kv, 16, hd]); every request is computed by itself."""
from __future__ import annotations

import numpy as np

PAGE = 16


def tokens(pool, blocks, h, n):
    """[n][hd]: the first n tokens of a request, kv head h, of pool [blocks][n_kv][16][hd]."""
    return pool[np.asarray(blocks), h].reshape(-1, pool.shape[-1])[:n]


def attention(q, k, v, page_table, ctx, nrow):
    """(out, lse, sum p |v|, largest sum |q k| / sqrt(hd)): [rows][n_q][hd], [rows][n_q], as out, as lse."""
    M, n_q, hd = q.shape
    n_kv = k.shape[1]
    G = n_q // n_kv
    out, mag = np.zeros_like(q), np.zeros_like(q)
    lse, big = np.zeros((M, n_q)), np.zeros((M, n_q))
    off = np.concatenate([[0], np.cumsum(nrow)])
    for b in range(len(ctx)):
        end = int(ctx[b]) + int(nrow[b])
        blocks = page_table[b, :(end + PAGE - 1) // PAGE]
        for h in range(n_kv):
            K, V = tokens(k, blocks, h, end), tokens(v, blocks, h, end)
            for j in range(int(nrow[b])):
                T, r, g = int(ctx[b]) + j + 1, off[b] + j, slice(h * G, (h + 1) * G)
                s = q[r, g] @ K[:T].T / np.sqrt(hd)
                m = s.max(-1, keepdims=True)
                p = np.exp(s - m)
                lse[r, g] = m[:, 0] + np.log(p.sum(-1))
                p /= p.sum(-1, keepdims=True)
                out[r, g], mag[r, g] = p @ V[:T], p @ np.abs(V[:T])
                big[r, g] = (np.abs(q[r, g]) @ np.abs(K[:T]).T).max(-1) / np.sqrt(hd)
    return out, lse, mag, big


def mass(q, k, lse, page_table, ctx, nrow, count, decay, prev):
    """(mass, sum of p x its relative error's unit, mask of the slots written) [blocks][n_kv][16]: prev is
    what was there (None: nothing); a page in several requests' tables gets all of theirs.  The second is sum
    p (sum |q k| / sqrt(hd) + |lse|)."""
    n_blocks, n_kv, _, hd = k.shape
    M, n_q, _ = q.shape
    G = n_q // n_kv
    got, err = np.zeros((n_blocks, n_kv, PAGE)), np.zeros((n_blocks, n_kv, PAGE))
    base, on = np.zeros_like(got), np.zeros(got.shape, bool)
    off = np.concatenate([[0], np.cumsum(nrow)])
    for b in range(len(ctx)):
        end = int(ctx[b]) + int(nrow[b])
        for t in range(end):
            blk, s = page_table[b, t // PAGE], t % PAGE
            on[blk, :, s] = True
            if t < ctx[b] and prev is not None:
                base[blk, :, s] = decay * prev[blk, :, s].astype(np.float64)
        n = int(nrow[b]) if count is None else int(np.clip(count[b], 0, nrow[b]))
        blocks = page_table[b, :(end + PAGE - 1) // PAGE]
        for h in range(n_kv):
            K = tokens(k, blocks, h, end)
            for j in range(n):
                T, r, g = int(ctx[b]) + j + 1, off[b] + j, slice(h * G, (h + 1) * G)
                p = np.exp(q[r, g] @ K[:T].T / np.sqrt(hd) - lse[r, g, None])
                e = p * (np.abs(q[r, g]) @ np.abs(K[:T]).T / np.sqrt(hd) + np.abs(lse[r, g, None]))
                for t in range(T):
                    got[blocks[t // PAGE], h, t % PAGE] += p[:, t].sum()
                    err[blocks[t // PAGE], h, t % PAGE] += e[:, t].sum()
    return base + got, err, on


def chosen(weight, keep, sink, recent):
    """Positions that stay of len(weight) tokens, in order."""
    n = len(weight)
    if keep >= n:
        return np.arange(n)
    w = np.where(np.isnan(weight), -np.inf, weight).astype(np.float64)
    middle = np.arange(sink, n - recent)
    # NaN is less than -infinity too
    order = np.lexsort((middle, -w[middle], np.isnan(weight[middle])))
    return np.sort(np.concatenate([np.arange(sink), middle[order[:keep - sink - recent]], np.arange(n - recent, n)])).astype(np.int64)


def evict(k, v, mass, page_table, ctx, keep, sink, recent, to_table, base):
    """k, v fp64 [layers][blocks][n_kv][16][hd] and mass [layers][blocks][n_kv][16], as they are after it, changed in
    place; returns (kept [layers][n_kv][total], |lo| + |hi| of every K element's pair, where a token was
    moved to, as k).  Everything is read before anything is written."""
    L, _, n_kv, _, hd = k.shape
    half = hd // 2
    freq = base ** (-2.0 * np.arange(half) / hd)
    kept = [[[] for _ in range(n_kv)] for _ in range(L)]
    pair = np.zeros_like(k)
    k0, v0, m0 = k.copy(), v.copy(), mass.copy()
    for l in range(L):
        for b in range(len(ctx)):
            n = min(int(keep[b]), int(ctx[b]))
            blocks = page_table[b]
            for h in range(n_kv):
                w = np.array([m0[l, blocks[t // PAGE], h, t % PAGE] for t in range(int(ctx[b]))], m0.dtype)
                src = chosen(w, n, int(sink[b]), int(recent[b]))
                kept[l][h].extend(src)
                for d, t in enumerate(src):
                    a, e = (blocks[t // PAGE], h, t % PAGE), (to_table[b][d // PAGE], h, d % PAGE)
                    lo, hi = k0[l][a][:half], k0[l][a][half:]
                    c, s = np.cos((d - t) * freq), np.sin((d - t) * freq)
                    k[l][e] = k0[l][a] if d == t else np.concatenate([lo * c - hi * s, hi * c + lo * s])
                    if d != t:
                        pair[l][e] = np.tile(np.abs(lo) + np.abs(hi), 2)
                    v[l][e], mass[l][e] = v0[l][a], m0[l][a]
    return np.array(kept, np.int32), pair
