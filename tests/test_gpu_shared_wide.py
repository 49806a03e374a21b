"""Attention over shared prefixes in work items of many turns: three and four row tiles on K and V in LDS, whose ring goes round
and whose block ids are asked for in several windows, in every instance; and batches of so much work that none is cut."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log, to_dev
from oracle import shared
from shared_harness import Case, attention_bounds
from test_gpu_shared import check_mass

pytestmark = pytest.mark.gpu


def heads(c, some):
    """The case's arrays of some kv heads: q, k, v."""
    G = c.n_q // c.n_kv
    q = c.q.reshape(c.M, c.n_kv, G, c.hd)[:, some].reshape(c.M, len(some) * G, c.hd)
    return q, c.k[:, some], c.v[:, some]


def check(c, some):
    kv, plan = c.pool(), c.plan()
    out, lse = c.run(kv, plan)
    again, lse2 = c.run(kv, plan)
    np.testing.assert_array_equal(out, again)
    np.testing.assert_array_equal(lse, lse2)
    G = c.n_q // c.n_kv
    q, k, v = heads(c, some)
    ref, rl, mag, big = shared.attention(q, k, v, c.pt, c.ctx, c.nrow)
    bo, bl = attention_bounds(ref, rl, mag, big, c.hd, int((c.ctx + c.nrow).max()), c.bf16)
    o = out.reshape(c.M, c.n_kv, G, c.hd)[:, some].reshape(ref.shape)
    l = lse.reshape(c.M, c.n_kv, G)[:, some].reshape(rl.shape)
    assert np.all(np.abs(o - ref) <= bo), (np.abs(o - ref) / bo).max()
    assert np.all(np.abs(l - rl) <= bl), (np.abs(l - rl) / bl).max()
    return kv, plan, lse


# head_dim, bf16, kv heads, tokens of the prefix: 64 rows of 64 query heads on each kv head, 32 bundles of four row tiles, with
# items of at least twice as many turns as there are stages in LDS
LONG = [(64, True, 8, 6144), (128, True, 8, 6144), (32, False, 8, 1280), (64, False, 8, 1280), (96, False, 4, 1024),
        (128, False, 4, 1024), (160, False, 4, 1024), (192, False, 4, 768), (224, False, 4, 768), (256, False, 4, 768)]


@pytest.mark.parametrize("hd,bf16,n_kv,prefix", LONG)
def test_many_rows_on_a_long_prefix(hd, bf16, n_kv, prefix):
    log(f"long items {hd} {bf16} {n_kv} {prefix}")
    c = Case([(prefix, [(3 + 5 * i, 4) for i in range(16)])], 64 * n_kv, n_kv, hd, bf16, seed=800 + hd)
    check(c, [0, n_kv // 2, n_kv - 1])


@pytest.mark.parametrize("hd,bf16", [(64, True), (128, True), (32, False), (256, False)])
def test_a_prompt_on_a_long_prefix(hd, bf16):
    """Rows of which each sees a token more: items whose last tiles are masked, on a prefix that its other request shares."""
    log(f"prompt {hd} {bf16}")
    c = Case([(1024, [(21, 70), (0, 5)])], 64, 1, hd, bf16, seed=830 + hd)
    check(c, [0])


def test_more_bundles_than_workgroups_stay_whole():
    """128 kv heads: four workgroups for each at a time, and 48 bundles, half of them of four row tiles over 65 tiles of tokens."""
    log("whole bundles")
    c = Case([(2080, [(7 + 3 * i, 2) for i in range(16)])] + [(0, [(90 + i, 2)]) for i in range(16)], 64 * 128, 128, 64, True, seed=840)
    some = [0, 63, 127]
    kv, plan, lse = check(c, some)
    mass = torch.zeros(c.k.shape[0], 128, 16, device="cuda")
    W.wisp_attention_mass(plan, kv, c.dev_q(), torch.from_numpy(lse).float().cuda(), mass)
    W.wisp_check(plan.ws)
    q, k, _ = heads(c, some)
    part = Sliced(c, q, k, len(some))
    got = mass[:, some].double().cpu().numpy()
    check_mass(part, got, lse.reshape(c.M, 128, 64)[:, some].reshape(c.M, -1), None, 1.0, None, np.zeros_like(got))


class Sliced:
    """What check_mass reads of a case."""

    def __init__(self, c, q, k, n_kv):
        self.q, self.k, self.pt, self.ctx, self.nrow, self.hd = q, k, c.pt, c.ctx, c.nrow, c.hd
        self.n_q, self.n_kv = q.shape[1], n_kv
