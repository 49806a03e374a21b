"""Attention over 8-bit pages whose scales reach the ends of what the cache holds, 2^-100 and 2^100, by
themselves and mixed within a request."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log
from kv8_harness import Case, attention_bound, dev, host_pool, shape
from oracle import kv8

pytestmark = pytest.mark.gpu

ENDS = {"least": (-100, -99), "largest": (99, 100), "both": (-100, 0, 100), "upper half": (50, 75, 100), "lower half": (-100, -75, -50)}
#          ctx, rows, query heads, kv heads, head_dim, bf16
SHAPES = [([1500, 3], [5, 3], 8, 2, 64, True), ([1500, 3], [5, 3], 8, 2, 64, False), ([700, 33], [9, 17], 32, 8, 128, True),
          ([40, 0], [200, 90], 8, 2, 128, True), ([100], [3], 3, 1, 224, False)]


@pytest.mark.parametrize("ends", ENDS)
@pytest.mark.parametrize("k", range(len(SHAPES)))
def test_scales_of_v_at_the_ends(k, ends):
    c = Case(*SHAPES[k], seed=60 + k).fill()
    c.scale[..., 1] = 2.0 ** np.random.default_rng(k).choice(ENDS[ends], c.scale.shape[:2])
    q = c.queries()
    kv, plan = c.pool(), c.plan()
    out = torch.full((c.M, c.n_q, c.hd), 7.0, dtype=torch.bfloat16 if c.bf16 else torch.float32, device="cuda")
    W.wisp_attention_kv8(plan, kv, dev(q, c.bf16), out)
    W.wisp_check(plan.ws)
    ref, mag, big = kv8.attention(q, *host_pool(kv), c.pt, c.ctx, c.nrow, c.n_kv)
    err = np.abs(out.double().cpu().numpy() - ref)
    tol = attention_bound(ref, mag, big, c.hd, int((c.ctx + c.nrow).max()), c.bf16)
    log(f"{SHAPES[k]}, V's scales {ENDS[ends]}: worst {np.max(err / tol):.3f} of its bound")
    assert np.all(err <= tol)


def _same_page(T, k_exp, v_exp, codes, n_q, hd, bf16, q):
    """Attention of one row to T tokens of one page, over and over."""
    m = W.GpuModel.shape_only(shape(n_q, 1, hd, bf16))
    pages = (T + 15) // 16
    kv = W.KV8Pool.zeros(1, 2, 1, hd)
    for pool, order, w in ((kv.k, kv8.k_order(hd), 0), (kv.v, kv8.v_order(hd), 1)):
        page = np.zeros(16 * hd, np.uint8)
        page[order.reshape(-1)] = kv8.e4m3_encode(np.broadcast_to(codes[w], (16, hd))).reshape(-1)
        pool.view(torch.uint8)[0, 1, 0] = torch.from_numpy(page).cuda()
    kv.scale[0, 1, 0] = torch.tensor([2.0 ** k_exp, 2.0 ** v_exp], device="cuda")
    desc = W.BatchDesc([T - 1], [0], torch.ones(1, pages, dtype=torch.int32, device="cuda"), 1.0)
    plan = W.wisp_kv8_plan(m, desc, W.workspace(W.wisp_kv8_workspace_size(m, desc)))
    x = torch.full((1, n_q, hd), q, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
    out = torch.empty_like(x)
    W.wisp_attention_kv8(plan, kv, x, out)
    W.wisp_check(plan.ws)
    return out.double().cpu().numpy()[0]


@pytest.mark.parametrize("bf16", [True, False], ids=["bf16", "f32"])
@pytest.mark.parametrize("v_exp,code", [(100, 448.0), (100, 2.0 ** -9), (-100, 448.0), (-100, 2.0 ** -9)])
@pytest.mark.parametrize("T", [17, 100003, 1 << 20])
def test_long_contexts_of_equal_tokens(T, v_exp, code, bf16):
    """Each result is the value that all tokens have: sums that pass fp32's range, or fall below it."""
    hd = 64
    v = np.where(np.arange(hd) % 3 == 0, -code, code)
    got = _same_page(T, 0, v_exp, (np.zeros(hd), v), 2, hd, bf16, 1.0)
    # the probabilities are equal, and with them both sums' errors but those of adding (sums of equal terms
    # in any order: 2^-24 of the sum for each of the log2(T) + 16 times that it grows by half)
    tol = 2.0 ** -8 if bf16 else (2 * 37 + 8) * 2.0 ** -24
    err = np.abs(got / (v * 2.0 ** v_exp) - 1).max()
    log(f"{T} tokens of {code} x 2^{v_exp}: off by {err:.2e}")
    assert err <= tol
