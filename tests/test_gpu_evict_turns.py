"""Evictions whose kept tokens take several turns of a workgroup, in every type and with 8 and 16 waves, in place and into other
pages; tokens that stay beside tokens that move; more requests than travel as arguments."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log
from test_gpu_evict import Cache

pytestmark = pytest.mark.gpu

# A turn has 64 tokens for each wave: 16 waves below 512 workgroups (requests x kv heads x layers x head_dim / 16), else 8
CASES = [
    # ctx, kv heads, head_dim, bf16, layers; keep; sink; recent
    ([3000, 70], 1, 32, False, 1, [2700, 33], [5, 0], [13, 3]),
    ([3100], 1, 64, False, 2, [2600], [40], [100]),
    ([2900], 1, 256, False, 1, [1500], [0], [0]),
    ([2500], 1, 160, False, 1, [2499], [3], [1]),             # one token leaves
    ([4000], 1, 64, True, 1, [3900], [0], [0]),               # nearly all stay: half pages all of kept tokens
    ([1300 + 7 * i for i in range(16)], 8, 64, True, 1, [520 + 50 * i for i in range(16)], [i for i in range(16)], [20] * 16),
    ([1200 + 9 * i for i in range(11)], 6, 128, False, 1, [1190 - 60 * i for i in range(11)], [16] * 11, [0] * 11),
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_kept_tokens_of_several_turns(case, in_place):
    ctx, n_kv, hd, bf16, layers, keep, sink, recent = CASES[case]
    log(f"turns {case} in place {in_place}")
    pages = (np.minimum(keep, ctx) + 15) // 16
    c = Cache(ctx, n_kv, hd, bf16, 900 + case, layers, spare=0 if in_place else int(pages.sum())).to_dev()
    to = None
    if not in_place:
        to = np.full((len(ctx), int(pages.max())), -1, np.int32)
        o = 0
        for i, n in enumerate(pages):
            to[i, :n] = c.free[o:o + n]
            o += int(n)
            to[i, :sink[i] // 16] = c.pt[i, :sink[i] // 16]
    kept = c.run(keep, sink, recent, to)
    c.check(kept, keep, sink, recent, to)


@pytest.mark.parametrize("bf16", [True, False])
@pytest.mark.parametrize("stay", [1, 7, 8, 9, 12, 16, 17, 31])
def test_tokens_that_stay_beside_tokens_that_move(bf16, stay):
    """The first `stay` tokens are the heaviest, the next one is the lightest: all behind it move up by one."""
    log(f"stay {stay} {bf16}")
    c = Cache([90, 40], 2, 64, bf16, 930 + stay)
    for b in range(2):
        for t in range(stay + 1):
            c.mass[:, c.pt[b, t // 16], :, t % 16] = 0.0 if t == stay else 1e6 + t
    c.to_dev()
    keep = [89, 39]
    kept = c.run(keep)
    assert (kept[0, 0, :stay] == np.arange(stay)).all() and kept[0, 0, stay] == stay + 1
    c.check(kept, keep)


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("n", [85, 86, 200])
def test_as_many_requests_as_arguments_hold_and_more(n, captured):
    log(f"requests {n} {captured}")
    ctx = 9 + 3 * np.arange(n) % 61
    c = Cache(ctx, 1, 64, True, 960 + n).to_dev()
    keep, sink, recent = (ctx // 2).tolist(), [1] * n, (ctx // 8).tolist()
    before = [t.clone() for t in (c.kv.k, c.kv.v, c.dm)]
    kept = torch.full((1, 1, int(np.sum(keep))), -9, dtype=torch.int32, device="cuda")
    ws = W.workspace(W.wisp_kv_evict_workspace_size(c.model, c.desc))
    call = lambda: W.wisp_kv_evict(c.model, c.kv, c.desc, keep, c.dm, kept, ws, sink, recent)
    if captured:
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            call()
        for _ in range(3):
            for t, x in zip((c.kv.k, c.kv.v, c.dm), before):
                t.copy_(x)
            kept.fill_(-9)
            ws.zero_()
            g.replay()
            torch.cuda.synchronize()
    else:
        call()
    W.wisp_check(ws)
    c.check(kept.cpu().numpy(), keep, sink, recent)
