"""wisp_verify_kv8 where the Q, K and V projection leaves several fp32 partial sums, which the append adds
up: each number of them that it has a kernel for, and numbers between. As the plain forward has it, over
the pages as they were written."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
import wisp_inputs as wi
from gpu_harness import gpu_model, log, to_dev
from test_gpu_verify_kv8 import _cache, _forward

pytestmark = pytest.mark.gpu

#         d_model, head_dim, query heads, kv heads, cached tokens, prompt rows, drafts, partial sums
CASES = [
    (1024, 64, 4, 2, [33], [0], [5], 2),
    (1536, 64, 8, 2, [33, 7, 100], [10, 0, 9], [9, 5, 4], 3),
    (2048, 128, 4, 1, [700], [0], [5], 4),
    (2560, 64, 4, 2, [0, 18], [20, 0], [3, 15], 5),
    (1536, 128, 4, 1, [0, 45], [180, 0], [5, 13], 6),
    (3584, 64, 8, 2, [15, 16, 17, 31], [0, 0, 0, 0], [9, 9, 9, 9], 7),
    (1024, 64, 4, 2, [5], [360], [9], 8),
    (8192, 64, 4, 2, [64, 3], [0, 0], [2, 1], 16),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_step_with_partial_sums(case):
    d, hd, n_q, n_kv, ctx, pre, gamma, splits = CASES[case]
    s = wi.ModelShape(f"one-layer-{d}", 1, d, n_q, n_kv, hd, 256, 256, "bf16", 10000.0)
    ctx, pre, gamma = (np.asarray(a, np.int32) for a in (ctx, pre, gamma))
    nrow = pre + gamma + 1
    plan = W.gemm_plan(int(nrow.sum()), (n_q + 2 * n_kv) * hd, d)
    log(f"d_model {d}, {int(nrow.sum())} rows: {plan}")
    assert plan["splits"] == splits
    rng = np.random.default_rng(40 + case)
    need = (ctx + nrow + 15) // 16
    perm, pt, o = rng.permutation(int(need.sum()) + 2).astype(np.int32), np.full((len(ctx), int(need.max()) + 1), -1, np.int32), 0
    for b, n in enumerate(need):
        pt[b, :n] = perm[o:o + n]
        o += n
    kv, gm = _cache(s, pt, ctx, len(perm), rng), gpu_model(s)
    desc = W.BatchDesc(ctx, gamma, to_dev(pt), 1.0, None, pre if pre.any() else None)
    tokens = rng.integers(0, s.vocab, desc.rows).astype(np.int32)
    ws = W.workspace(W.wisp_verify_kv8_workspace_size(gm.c, desc))
    acc = torch.empty(desc.B, dtype=torch.int32, device="cuda")
    out = torch.empty(desc.M, dtype=torch.int32, device="cuda")
    logits = torch.full((desc.M, s.vocab), float("nan"), device="cuda")
    q = torch.full((desc.S, s.vocab), 1.0 / s.vocab, device="cuda")
    W.wisp_verify_kv8(gm.c, kv, desc, to_dev(tokens), q, 5, acc, out, logits, ws)
    W.wisp_check(ws)
    ref = _forward(s, kv, pt, ctx, nrow, tokens, True)      # checks the new rows' pages
    ref = ref[np.concatenate([np.arange(e - g - 1, e) for e, g in zip(np.cumsum(nrow), gamma)])]
    # a row is rounded to bf16 seven times on its way (two norms, queries, probabilities, heads, the MLP's
    # product, the last norm): 2^-8 each of its scale, and as much for all fp32 sums
    err = np.abs(logits.cpu().numpy() - ref) / np.abs(ref).max(-1, keepdims=True)
    log(f"  logits off by {err.max():.2e} of their row's largest")
    assert err.max() <= 8 * 2.0 ** -8
