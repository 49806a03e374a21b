"""Scores and log-sum-exps of infinity in attention over shared prefixes and in its weights: rows whose tokens the waves share, on K
and V in LDS, in results of several parts."""
import numpy as np
import pytest

from oracle import shared
from shared_harness import Case, attention_bounds
from test_gpu_shared_ranges import CASES, weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [np.inf, -np.inf])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_scores_of_infinity(case, bad):
    """An infinite key in a common (or early) token, seen by every row of its requests: a row is NaN where its score is +infinity and
    as without that token where it is -infinity."""
    c = Case(*CASES[case], seed=740 + case)
    c.k[c.pt[0, 0], 0, 7, 5] = 0.0
    big = shared.attention(c.q, c.k, c.v, c.pt, c.ctx, c.nrow)[3]
    c.k[c.pt[0, 0], 0, 7, 5] = bad
    G = c.n_q // c.n_kv
    sees = np.zeros((c.M, c.n_q), bool)
    for b in range(len(c.ctx)):
        if c.pt[b, 0] == c.pt[0, 0]:
            sees[c.off[b]:c.off[b + 1], :G] = True
    nan = sees & (c.q[..., 5] * bad > 0)
    assert nan.any() and (sees & ~nan).any()
    kv, plan = c.pool(), c.plan()
    out, lse = c.run(kv, plan)
    with np.errstate(invalid="ignore"):
        ref, rl, mag, _ = shared.attention(c.q, c.k, c.v, c.pt, c.ctx, c.nrow)
    bo, bl = attention_bounds(ref, rl, mag, big, c.hd, int((c.ctx + c.nrow).max()), c.bf16)
    assert np.isnan(out[nan]).all() and np.isnan(lse[nan]).all()
    assert np.all((np.abs(out - ref) <= bo)[~nan]) and np.all((np.abs(lse - rl) <= bl)[~nan])


@pytest.mark.parametrize("case", range(len(CASES)))
def test_rows_with_an_lse_of_infinity_add_nothing(case):
    c = Case(*CASES[case], seed=760 + case)
    kv, plan = c.pool(), c.plan()
    _, lse = c.run(kv, plan)
    count = np.maximum(c.nrow - 1, 0).astype(np.int32)
    gone = lse.copy()
    gone[c.off[1:] - 1] = np.inf                              # the last row of each request
    np.testing.assert_array_equal(weights(c, kv, plan, gone), weights(c, kv, plan, lse, count))
