"""A common prefix in the page manager: a session of its own, named in every reservation, whose pages stand in front of the
other sessions' in their tables."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import to_dev
from shared_harness import Case
from test_gpu_shared_steps import evict, step

pytestmark = pytest.mark.gpu

PREFIX, COMMON, STRIDE = 48, 1000, 40


def tables(mgr, own):
    """Page tables of the sessions 1, 2, .. of `own` tokens behind the prefix."""
    sids = [COMMON] + list(range(1, len(own) + 1))
    t, evicted = mgr.reserve(sids, [PREFIX] + list(own), STRIDE)
    assert evicted == 0
    n = PREFIX // 16
    return np.concatenate([np.tile(t[0, :n], (len(own), 1)), t[1:, :STRIDE - n]], 1).astype(np.int32)


@pytest.mark.parametrize("bf16", [True, False])
def test_sessions_behind_a_prefix_that_is_a_session(bf16):
    own, rows = np.array([300, 120, 77]), np.array([3, 1, 2])
    c = Case([(PREFIX, list(zip(own, rows)))], 8, 2, 64, bf16, seed=88)
    mgr = W.KVManager(64)
    pt = tables(mgr, own + rows)
    k, v = (np.full((64,) + c.k.shape[1:], np.nan) for _ in range(2))
    for i in range(3):
        n = int(c.ctx[i] + rows[i] + 15) // 16
        k[pt[i, :n]], v[pt[i, :n]] = c.k[c.pt[i, :n]], c.v[c.pt[i, :n]]
    c.k, c.v, c.pt = k, v, pt
    c.desc = W.BatchDesc(c.ctx, c.gamma, to_dev(pt))
    mgr.commit([COMMON], [PREFIX])
    kv, mass = c.pool(), torch.zeros(64, 2, 16, device="cuda")
    step(c, kv, mass, c.nrow, 1.0)
    # the rows are in the cache now; the prefix and the last 16 stay, and the most attended of the others
    c.ctx = c.ctx + c.nrow
    keep = np.array([PREFIX + 100, PREFIX + 33, PREFIX + 79], np.int32)      # of the third all stay
    first = c.k[pt[0, :PREFIX // 16]].copy()
    evict(c, kv, mass, keep, np.full(3, PREFIX), np.full(3, 16))
    np.testing.assert_array_equal(c.k[pt[0, :PREFIX // 16]], first)
    left = np.minimum(keep, c.ctx) - PREFIX
    mgr.commit([1, 2, 3], left)
    assert mgr.stats()["free_pages"] == 64 - int(((left + 15) // 16).sum()) - PREFIX // 16
    # the next step's rows, as the model would have stored them, on the same pages and new ones
    c.nrow = np.array([2, 4, 1], np.int32)
    again = tables(mgr, left + c.nrow)
    for i in range(3):
        n = (int(left[i]) + 15) // 16 + PREFIX // 16
        np.testing.assert_array_equal(again[i, :n], pt[i, :n])
    c.pt, c.ctx, c.gamma = again, (left + PREFIX).astype(np.int32), c.nrow - 1
    for i in range(3):
        for t in range(int(c.ctx[i]), int(c.ctx[i] + c.nrow[i])):
            for pool in (c.k, c.v):
                pool[c.pt[i, t // 16], :, t % 16] = c.round(c.rng.normal(0, 1.15, (2, 64)))
    c.M, c.off = int(c.nrow.sum()), np.concatenate([[0], np.cumsum(c.nrow)])
    c.q = c.round(c.rng.normal(0, 1.15, (c.M, 8, 64)))
    c.desc = W.BatchDesc(c.ctx, c.gamma, to_dev(c.pt))
    step(c, c.pool(), mass, c.nrow, 0.9)
