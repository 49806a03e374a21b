"""Attention over shared prefixes on bf16 rows of which a few tokens have most: what the rounding of probabilities leaves."""
import numpy as np
import pytest

from gpu_harness import log
from oracle import shared
from shared_harness import HALF, U, Case

pytestmark = pytest.mark.gpu

# groups of (prefix, [(own cached tokens, rows)]), query heads, kv heads, head_dim
CASES = [
    ([(64, [(9, 3), (40, 2)]), (0, [(140, 5)])], 4, 2, 64),
    ([(1024, [(64, 5), (9, 2)])], 32, 8, 128),
    ([(512, [(40, 40), (9, 33), (0, 30)])], 8, 2, 128),
    ([(2048, [(3 + 5 * i, 4) for i in range(8)])], 128, 2, 64),
]


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_a_row_divides_by_the_probabilities_that_multiplied_v(case, bad):
    """out = sum p v / sum p over probabilities that are each off by half a step: what they are off by counts as far as V differs from
    the result.  So a token with nearly all of a row gives its V, rounded once.  (bad: V of the last new token holds an infinity in a dim
    of kv head 0, which the rows before it must not touch.)"""
    log(f"rounding {CASES[case]} {bad}")
    c = Case(*CASES[case], bf16=True, seed=950 + case, std=2.5)
    unseen = []
    if bad:
        for b in range(len(c.ctx)):
            t = int(c.ctx[b] + c.nrow[b]) - 1
            c.v[c.pt[b, t // 16], 0, t % 16, 3] = np.inf
            unseen.append(c.off[b + 1] - 1)                   # the row that does see it
    out, lse = c.run()
    _, rl, mag, big = shared.attention(c.q, c.k, np.nan_to_num(c.v, posinf=0.0), c.pt, c.ctx, c.nrow)
    G, h = c.n_q // c.n_kv, HALF[True]
    worst = 0.0
    for b in range(len(c.ctx)):
        end = int(c.ctx[b] + c.nrow[b])
        for g in range(c.n_kv):
            K, V = (shared.tokens(p, c.pt[b, :(end + 15) // 16], g, end) for p in (c.k, c.v))
            for j in range(int(c.nrow[b])):
                r, n, hs = c.off[b] + j, int(c.ctx[b]) + j + 1, slice(g * G, (g + 1) * G)
                if r in unseen:
                    continue
                w = np.exp(c.q[r, hs] @ K[:n].T / np.sqrt(c.hd) - rl[r, hs, None])
                ref = w @ V[:n]
                apart = (w[:, :, None] * np.abs(V[None, :n] - ref[:, None])).sum(1)
                # fp32: the exponent by (hd + 8) half steps of the score's terms, the sums by T + 256, twice
                rest = 2 * ((c.hd + 8) * U * np.maximum(big[r, hs], 1.0) + (n + 256) * U)[:, None] * mag[r, hs]
                bound = h * np.abs(ref) + (h / (1 - h) * apart + rest) * (1 + h)
                worst = max(worst, (np.abs(out[r, hs] - ref) / bound).max())
    assert worst <= 1.0, worst
