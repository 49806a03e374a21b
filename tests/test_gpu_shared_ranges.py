"""Attention over shared prefixes and the weights it gives, with scores so large that roundings show in their differences."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log, to_dev
from oracle import shared
from shared_harness import HALF, U, Case

pytestmark = pytest.mark.gpu

LOG2E = 1.4426950408889634

# groups of (prefix, [(own cached tokens, rows)]), query heads, kv heads, head_dim, bf16: the waves of a row tile share its
# tokens; three and four row tiles on K and V in LDS; results in parts; three query heads per kv head
CASES = [
    ([(32, [(9, 3), (4, 2)]), (0, [(40, 5)])], 4, 2, 64, True),
    ([(32, [(9, 3), (4, 2)]), (0, [(40, 5)])], 4, 2, 64, False),
    ([(256, [(40, 40), (9, 33), (0, 30)])], 8, 2, 128, True),
    ([(256, [(40, 40), (9, 33)])], 4, 2, 64, False),
    ([(1024, [(40, 5), (9, 2)])], 6, 2, 64, True),
    ([(288, [(40, 60), (70, 3)])], 4, 2, 96, False),
]


def exact_scores(case, seed, power):
    """A case whose products q . k are whole numbers below 2^24, exact in fp32 in any order: 2^power, -2^power or 0 by
    the row, and up to 27 on either side."""
    c = Case(*case, seed=seed)
    sign = np.array([1.0, 0.0, -1.0, 1.0])[np.arange(c.M) % 4]
    c.q[:] = 0.0
    c.q[..., 0] = (sign * 2.0 ** (power - power // 2))[:, None]
    c.q[..., 1:4] = c.rng.integers(-3, 4, c.q.shape[:2] + (3,))
    there = ~np.isnan(c.k)
    c.k[there] = 0.0
    c.k[..., 0] = np.where(there[..., 0], 2.0 ** (power // 2), np.nan)
    c.k[..., 1:4] = np.where(there[..., 1:4], c.rng.integers(-3, 4, c.k.shape[:3] + (3,)), np.nan)
    return c


def weights(c, kv, plan, lse, count=None):
    m = torch.zeros(c.k.shape[0], c.n_kv, 16, device="cuda")
    W.wisp_attention_mass(plan, kv, c.dev_q(), torch.from_numpy(lse).float().cuda(), m, None, 1.0, None if count is None else to_dev(count))
    W.wisp_check(plan.ws)
    return m.double().cpu().numpy()


@pytest.mark.parametrize("power", [18, 20, 23])              # of q . k: scores of 2^15 to 2^20 (head_dim 64)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_large_scores_that_differ_by_little(case, power):
    """The scores themselves are exact, so what is left is what the sizes of the maximum, of lse and of a score bring."""
    log(f"large scores {CASES[case]} 2^{power}")
    c = exact_scores(CASES[case], 700 + case, power)
    kv, plan = c.pool(), c.plan()
    out, lse = c.run(kv, plan)
    ref, rl, mag, _ = shared.attention(c.q, c.k, c.v, c.pt, c.ctx, c.nrow)
    # Differences of scores are exact; their factor (four roundings of a difference of up to 54 / 8 x log2 e, 40 half steps), the
    # exponential and the parts are 64 roundings, the sum T + 256.  Up to 65536 / log2(e) a maximum times that factor is rounded
    # as well, once for each part: one half step of it.  lse: a factor of two roundings, the product's and the sum's.
    sums, T = 64 + 256, int((c.ctx + c.nrow).max())
    part = np.where(np.abs(rl) * LOG2E <= 65536, np.abs(rl), 0.0) * U
    bound = HALF[c.bf16] * np.abs(ref) + ((HALF[True] if c.bf16 else 0.0) + 4 * part + 2 * (T + sums) * U)[..., None] * mag * (1 + HALF[c.bf16])
    assert np.all(np.abs(out - ref) <= bound), (np.abs(out - ref) / bound).max()
    bl = 5 * U * np.abs(rl) + (T + sums) * U
    assert np.all(np.abs(lse - rl) <= bl), (np.abs(lse - rl) / bl).max()
    # a weight: 2^-21 |lse| of its exponent, and its part in the sums
    off = np.expm1(2.0 ** -21 * np.abs(rl))
    for count in (None, c.rng.integers(0, c.nrow + 1).astype(np.int32)):
        got = weights(c, kv, plan, lse, count)
        want, _, on = shared.mass(c.q, c.k, rl, c.pt, c.ctx, c.nrow, count, 1.0, None)
        room = np.zeros_like(want)
        for b in range(len(c.ctx)):
            end = int(c.ctx[b] + c.nrow[b])
            for h in range(c.n_kv):
                K = shared.tokens(c.k, c.pt[b, :(end + 15) // 16], h, end)
                for j in range(int(c.nrow[b] if count is None else count[b])):
                    n, r, g = int(c.ctx[b]) + j + 1, c.off[b] + j, slice(h * c.n_q // c.n_kv, (h + 1) * c.n_q // c.n_kv)
                    p = np.exp(c.q[r, g] @ K[:n].T / np.sqrt(c.hd) - rl[r, g, None]) * off[r, g, None]
                    np.add.at(room, (c.pt[b, np.arange(n) // 16], h, np.arange(n) % 16), p.sum(0))
        bound = room * (1 + 2.0 ** -10) + (c.M * c.n_q // c.n_kv + 128) * U * want
        assert np.all((np.abs(got - want) <= bound)[on]), np.nanmax((np.abs(got - want) / bound)[on])


@pytest.mark.parametrize("power", [20, 26, 27, 31, 60, 120])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_one_token_that_has_all_of_a_row(case, power):
    """Scores of 2^power / sqrt(head_dim), that of one token a quarter above: its V is the result and its weight 1, exactly, at any
    size.  Every fourth row has scores of zero, and of each request some rows do not count."""
    log(f"one token {CASES[case]} 2^{power}")
    c = Case(*CASES[case], seed=720 + case)
    c.q[:] = 0.0
    plain = np.arange(c.M) % 4 == 3
    c.q[..., 0] = np.where(plain, 0.0, 2.0 ** (power - power // 2))[:, None]
    there = ~np.isnan(c.k)
    c.k[there] = 0.0
    c.k[..., 0] = np.where(there[..., 0], 2.0 ** (power // 2), np.nan)
    top = []                                                  # of each request: the position
    for b in range(len(c.ctx)):
        top.append(int(c.ctx[b]) if b % 2 else 5 if c.pt[b, 0] == c.pt[0, 0] else 3)   # its first new token, or an early one
        c.k[c.pt[b, top[b] // 16], :, top[b] % 16, 0] = 2.0 ** (power // 2) * (1.5 if b % 2 else 1.25)
    kv, plan = c.pool(), c.plan()
    out, lse = c.run(kv, plan)
    count = np.maximum(c.nrow - 1, 1).astype(np.int32)
    got = weights(c, kv, plan, lse, count)
    want, flat = np.zeros_like(got), np.zeros_like(got)       # what the tops have, and what rows of equal scores give
    G = c.n_q // c.n_kv
    for b in range(len(c.ctx)):
        for j in range(int(c.nrow[b])):
            r, n = c.off[b] + j, int(c.ctx[b]) + j + 1
            if plain[r]:
                if j < count[b]:
                    at = np.arange(n)
                    np.add.at(flat, (c.pt[b, at // 16], slice(None), at % 16), G / n)
                continue
            for h in range(c.n_kv):
                v = c.v[c.pt[b, top[b] // 16], h, top[b] % 16]
                np.testing.assert_array_equal(out[r, h * G:(h + 1) * G], np.tile(v, (G, 1)))
                if j < count[b]:
                    want[c.pt[b, top[b] // 16], h, top[b] % 16] += G
    # equal scores: an exponent of their number's logarithm (below 12, two roundings), the sums' order
    assert np.all(np.abs(got - want - flat) <= (want + flat) * (c.M * G + 128) * U), np.abs(got - want - flat).max()
