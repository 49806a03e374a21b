"""The 8-bit KV cache in fp64 numpy: e4m3 codes, page order, append and attention (test
infrastructure; written from the definitions in include/wisp.h)."""
from __future__ import annotations

import numpy as np

PAGE = 16
E4M3_MAX = 448.0
NAN_CODE = 0x7F


def e4m3_values() -> np.ndarray:
    """fp64 value of each of the 256 codes (1 sign, 4 exponent bits of bias 7, 3 mantissa bits)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


VALUES = e4m3_values()
_POS = VALUES[:127]


def e4m3_encode(x) -> np.ndarray:
    """Nearest code, ties to the even one; |x| <= 448, NaN to the NaN code."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    i = np.clip(np.searchsorted(_POS, np.nan_to_num(a)), 1, 126)
    lo, hi = a - _POS[i - 1], _POS[i] - a
    i = np.where((lo < hi) | ((lo == hi) & (i % 2 == 1)), i - 1, i)
    c = np.where(np.signbit(x), i + 128, i).astype(np.uint8)
    return np.where(np.isnan(x), NAN_CODE, c).astype(np.uint8)


def k_order(hd: int) -> np.ndarray:
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return (((e // 32) * 4 + (e % 32) // 8) * 8 + (s // 8) * 4 + s % 4) * 16 + ((s // 4) % 2) * 8 + e % 8


def v_order(hd: int) -> np.ndarray:
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return ((e // 32) * 2 + s // 8) * 256 + (e % 16) * 16 + ((e // 16) % 2) * 8 + s % 8


def scale_of(most) -> float:
    """2^k, the smallest k >= -100 with most <= 448 * 2^k; 1 for most = 0."""
    if most == 0:
        return 1.0
    k = -100
    while most > E4M3_MAX * 2.0 ** k:
        k += 1
    return 2.0 ** k


def rotate(x, pos, base):
    """x [rows][heads][hd] rotated by pos [rows] (rotate-half pairs), fp64."""
    hd = x.shape[-1]
    a = pos[:, None, None] * base ** (-2.0 * np.arange(hd // 2) / hd)
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1)


def append(k, v, scale, page_table, ctx, nrow, qkv, n_q, n_kv, hd, base):
    """k, v uint8 [blocks][n_kv][16 * hd], scale [blocks][n_kv][2], changed in place; qkv fp64
    [rows][(n_q + 2 n_kv) * hd].  Returns (rotated q fp64, unquantised K, V [rows][n_kv][hd])."""
    x = qkv.reshape(qkv.shape[0], n_q + 2 * n_kv, hd)
    pos = np.concatenate([c + np.arange(n) for c, n in zip(ctx, nrow)]).astype(np.float64)
    with np.errstate(invalid="ignore"):
        q, kn = rotate(x[:, :n_q], pos, base), rotate(x[:, n_q:n_q + n_kv], pos, base)
    vn = x[:, n_q + n_kv:]
    off = np.concatenate([[0], np.cumsum(nrow)])
    orders = (k_order(hd), v_order(hd))
    limit = E4M3_MAX * 2.0 ** 100
    for b in range(len(ctx)):
        end = int(ctx[b]) + int(nrow[b])
        for p in range(int(ctx[b]) // PAGE, (end + PAGE - 1) // PAGE):
            blk = page_table[b, p]
            held = min(max(int(ctx[b]) - p * PAGE, 0), PAGE)
            filled = min(end - p * PAGE, PAGE)
            r0 = off[b] + p * PAGE + held - int(ctx[b])
            for h in range(n_kv):
                new = [t[r0:r0 + filled - held, h] for t in (kn, vn)]
                with np.errstate(invalid="ignore"):
                    bad = ~(np.all(np.abs(new[0]) <= limit, -1) & np.all(np.abs(new[1]) <= limit, -1))
                    bad |= ~np.all(np.isfinite(x[r0:r0 + filled - held, n_q + h]), -1)
                for w, (pool, order) in enumerate(zip((k, v), orders)):
                    val = VALUES[pool[blk, h][order]] * scale[blk, h, w]
                    val[held:filled] = new[w]
                    val[held:filled][bad] = np.nan if w == 0 else 0.0
                    ok = val[:filled][~np.isnan(val[:filled])]
                    sc = scale_of(np.abs(ok).max() if ok.size else 0.0)
                    page = pool[blk, h].copy()
                    page[order[:filled]] = e4m3_encode(val[:filled] / sc)
                    pool[blk, h] = page
                    scale[blk, h, w] = sc
    return q, kn, vn


def tokens(pool, scale, which: str, blocks, h: int, T: int, hd: int) -> np.ndarray:
    """fp64 values [T][hd] of the first T tokens in the pages `blocks` of kv head h."""
    order = (k_order if which == "k" else v_order)(hd)
    val = VALUES[pool[blocks, h][:, order]] * scale[blocks, h, 0 if which == "k" else 1][:, None, None]
    return val.reshape(-1, hd)[:T]


def attention(q, k, v, scale, page_table, ctx, nrow, n_kv):
    """(out, sum p |v|, largest sum |q k| / sqrt(hd)): fp64 [rows][n_q][hd], the same, [rows][n_q]."""
    M, n_q, hd = q.shape
    G = n_q // n_kv
    out, mag, big = np.zeros_like(q), np.zeros_like(q), np.zeros((M, n_q))
    off = np.concatenate([[0], np.cumsum(nrow)])
    for b in range(len(ctx)):
        end = int(ctx[b]) + int(nrow[b])
        blocks = page_table[b, :(end + PAGE - 1) // PAGE]
        for h in range(n_kv):
            K, V = (tokens(p, scale, w, blocks, h, end, hd) for p, w in ((k, "k"), (v, "v")))
            for j in range(int(nrow[b])):
                T = int(ctx[b]) + j + 1
                qq = q[off[b] + j, h * G:(h + 1) * G]
                s = qq @ K[:T].T / np.sqrt(hd)
                p = np.exp(s - s.max(-1, keepdims=True))
                p /= p.sum(-1, keepdims=True)
                out[off[b] + j, h * G:(h + 1) * G] = p @ V[:T]
                mag[off[b] + j, h * G:(h + 1) * G] = p @ np.abs(V[:T])
                big[off[b] + j, h * G:(h + 1) * G] = (np.abs(qq) @ np.abs(K[:T]).T).max(-1) / np.sqrt(hd)
    return out, mag, big
