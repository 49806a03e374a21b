"""wisp_verify_kv8, the whole step on the 8-bit cache: the pages it writes and its logits against a
plain fp64 forward, its decisions against the oracle's on the same logits, and what the tokens'
log probabilities (wisp_token_logprobs) say afterwards, as a server would run them.

The forward attends to the pages as the GPU wrote them, each of which is checked on its own: a
code next to a border may fall on either side of it, and would otherwise move all that follows."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
import wisp_inputs as wi
from gpu_harness import check_decisions_on_gpu_logits, gpu_model, log, rel_row_err, to_dev
from kv8_harness import host_pool
from oracle import kv8

pytestmark = pytest.mark.gpu

MINI_BF16 = wi.ModelShape("mini-bf16-gqa", 2, 256, 8, 2, 64, 512, 1024, "bf16", 10000.0)
WIDE_BF16 = wi.ModelShape("mini-bf16-128", 2, 512, 8, 2, 128, 512, 1024, "bf16", 500000.0)
F32_32 = wi.ModelShape("mini-f32-32", 2, 128, 4, 1, 32, 256, 512, "f32", 10000.0)


def _cache(s, pt, ctx, n_blocks, rng):
    """Seeded pages of the cached contexts; NaN codes everywhere else."""
    shp = (s.n_layers, n_blocks, s.n_kv_heads, 16 * s.head_dim)
    pools = [np.full(shp, kv8.NAN_CODE, np.uint8) for _ in range(2)]
    scale = np.full(shp[:3] + (2,), np.nan, np.float32)
    for b, n in enumerate(ctx):
        for p in range((int(n) + 15) // 16):
            held = min(int(n) - 16 * p, 16)
            for l in range(s.n_layers):
                for pool, order in zip(pools, (kv8.k_order(s.head_dim), kv8.v_order(s.head_dim))):
                    page = pool[l, pt[b, p]].copy()
                    page[:, order[:held].reshape(-1)] = kv8.e4m3_encode(
                        np.clip(rng.normal(0, 90, (s.n_kv_heads, held * s.head_dim)), -448, 448))
                    pool[l, pt[b, p]] = page
                scale[l, pt[b, p]] = 2.0 ** -8
    f8 = lambda a: torch.from_numpy(a).cuda().view(torch.float8_e4m3fn)
    return W.KV8Pool(f8(pools[0]), f8(pools[1]), torch.from_numpy(scale).cuda())


def _f64(t):
    return t.double().cpu().numpy()


def _forward(s, kv, pt, ctx, nrow, tokens, bf16):
    """fp64 logits of every row over the pages of kv, checking the new rows' K and V in them."""
    g = wi.global_weights(s, device="cpu")
    rms = lambda x, w: x / np.sqrt((x * x).mean(-1, keepdims=True) + s.rms_eps) * w
    pos = np.concatenate([c + np.arange(n) for c, n in zip(ctx, nrow)]).astype(np.float64)
    off = np.concatenate([[0], np.cumsum(nrow)])
    h = _f64(g["embed"])[tokens]
    for l in range(s.n_layers):
        w = {k: _f64(v) for k, v in wi.layer_weights(s, l, device="cpu").items()}
        x = rms(h, w["attn_norm"])
        heads = lambda m, n: (x @ w[m].T).reshape(len(tokens), n, s.head_dim)
        q = kv8.rotate(heads("wq", s.n_q_heads), pos, s.rope_base)
        new = (kv8.rotate(heads("wk", s.n_kv_heads), pos, s.rope_base), heads("wv", s.n_kv_heads))
        k, v, sc = host_pool(kv.layer(l))
        for b in range(len(ctx)):
            end = int(ctx[b] + nrow[b])
            blocks = pt[b, :(end + 15) // 16]
            for hd in range(s.n_kv_heads):
                for pool, which, n in ((k, "k", new[0]), (v, "v", new[1])):
                    got = kv8.tokens(pool, sc, which, blocks, hd, end, s.head_dim)[int(ctx[b]):]
                    want = n[off[b]:off[b + 1], hd]
                    page = np.repeat(sc[blocks, hd, 0 if which == "k" else 1], 16)[int(ctx[b]):end, None]
                    # half a step of e4m3, and what the activations' own rounding moves: fp32 sums,
                    # or two roundings of bf16 at the row's scale
                    slack = (2.0 ** -6 if bf16 else 2.0 ** -16) * np.abs(want).max(-1, keepdims=True)
                    assert np.all(np.abs(got - want) <= 2.0 ** -4 * (np.abs(want) + slack) + 2.0 ** -10 * page + slack), (l, b, hd, which)
        o, _, _ = kv8.attention(q, k, v, sc, pt, ctx, nrow, s.n_kv_heads)
        h = h + o.reshape(len(tokens), -1) @ w["wo"].T
        x = rms(h, w["mlp_norm"])
        gate, up = x @ w["w_gate"].T, x @ w["w_up"].T
        h = h + (gate / (1 + np.exp(-gate)) * up) @ w["w_down"].T
    return rms(h, _f64(g["final_norm"])) @ _f64(g["lm_head"]).T


CASES = [
    (wi.TINY, [37, 0, 90, 15, 120, 3], [4, 16, 2, 0, 7, 1], None),
    (wi.TINY, [0, 50, 0], [3, 1, 0], [40, 0, 5]),
    (F32_32, [33, 5], [2, 3], None),
    (MINI_BF16, [37, 0, 90, 15, 120, 3], [4, 16, 2, 0, 7, 1], None),
    (MINI_BF16, [0, 50, 16], [3, 1, 0], [70, 0, 5]),
    (WIDE_BF16, [700, 9], [5, 8], None),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_step_matches_a_plain_forward(case):
    s, ctx, gamma, pre = CASES[case]
    ctx, gamma = np.asarray(ctx, np.int32), np.asarray(gamma, np.int32)
    pre_ = np.zeros_like(ctx) if pre is None else np.asarray(pre, np.int32)
    nrow = pre_ + gamma + 1
    log(f"{s.name}: ctx={ctx.tolist()} gamma={gamma.tolist()} prompt={pre_.tolist()}")
    rng = np.random.default_rng(900 + case)
    need = (ctx + nrow + 15) // 16
    perm, pt, o = rng.permutation(int(need.sum()) + 2).astype(np.int32), np.full((len(ctx), int(need.max()) + 1), -1, np.int32), 0
    for b, n in enumerate(need):
        pt[b, :n] = perm[o:o + n]
        o += n
    kv = _cache(s, pt, ctx, len(perm), rng)
    gm = gpu_model(s)
    desc = W.BatchDesc(ctx, gamma, to_dev(pt), 1.0, None, pre)
    tokens = rng.integers(0, s.vocab, desc.rows).astype(np.int32)
    q = torch.softmax(2.0 * torch.randn(max(desc.S, 1), s.vocab, generator=torch.Generator().manual_seed(case)), -1)
    ws = W.workspace(W.wisp_verify_kv8_workspace_size(gm.c, desc))
    acc = torch.full((desc.B,), -7, dtype=torch.int32, device="cuda")
    out = torch.full((desc.M,), -7, dtype=torch.int32, device="cuda")
    logits = torch.full((desc.M, s.vocab), float("nan"), device="cuda")
    dq, dt = q.cuda(), to_dev(tokens)
    W.wisp_verify_kv8(gm.c, kv, desc, dt, dq, 5, acc, out, logits, ws)
    W.wisp_check(ws)
    ref = _forward(s, kv, pt, ctx, nrow, tokens, s.dtype == "bf16")
    vrow = np.concatenate([np.arange(e - g - 1, e) for e, g in zip(np.cumsum(nrow), gamma)])
    got = logits.cpu().numpy().astype(np.float64)
    if s.dtype == "bf16":
        worst = np.abs(got - ref[vrow]).max()
        assert worst <= 2e-2, worst
    else:
        worst = rel_row_err(got, ref[vrow]).max()
        assert worst <= 1e-4, worst
    log(f"  logits off by {worst:.2e}")
    check_decisions_on_gpu_logits(acc.cpu().numpy(), out.cpu().numpy(), logits.cpu().numpy(), tokens[vrow], q[:desc.S].numpy(),
                                  gamma, 1.0, 5)
    # the same outputs without a logits buffer, and repeated
    ws2 = W.workspace(W.wisp_verify_kv8_workspace_size(gm.c, desc) + W.wisp_logits_workspace_size(gm.c, desc))
    acc2, out2 = torch.empty_like(acc), torch.empty_like(out)
    before = [kv.k.view(torch.uint8).clone(), kv.v.view(torch.uint8).clone(), kv.scale.clone()]
    W.wisp_verify_kv8(gm.c, kv, desc, dt, dq, 5, acc2, out2, None, ws2)
    W.wisp_check(ws2)
    assert torch.equal(acc, acc2) and torch.equal(out, out2)
    for a, b in zip(before, (kv.k.view(torch.uint8), kv.v.view(torch.uint8), kv.scale)):
        assert torch.equal(torch.nan_to_num(a.float(), 7.0), torch.nan_to_num(b.float(), 7.0))
    # what the answer says about its tokens: padding rows (-1) are passed over
    lp = torch.full((desc.M,), 9.0, device="cuda")
    ids, tlp = torch.zeros(desc.M, 3, dtype=torch.int32, device="cuda"), torch.zeros(desc.M, 3, device="cuda")
    W.wisp_token_logprobs(logits, s.vocab, out, 1.0, lp, None, ids, tlp)
    want = torch.log_softmax(logits.double(), -1)
    on = out >= 0
    assert (lp[~on] == 9.0).all()
    assert (lp[on].double() - want[on, out[on].long()]).abs().max() <= 2.0 ** -20 * want.abs().max()
    assert torch.equal(ids[on].long(), torch.sort(logits[on], dim=-1, descending=True, stable=True)[1][:, :3])


def test_refusals_of_the_step():
    s = MINI_BF16
    gm = gpu_model(s)
    desc = W.BatchDesc([20], [2], torch.zeros(1, 2, dtype=torch.int32, device="cuda"), 1.0)
    kv = W.KV8Pool.zeros(s.n_layers, 4, s.n_kv_heads, s.head_dim)
    t = torch.zeros(3, dtype=torch.int32, device="cuda")
    q = torch.full((2, s.vocab), 1.0 / s.vocab, device="cuda")
    a, o = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    ws = W.workspace(W.wisp_verify_kv8_workspace_size(gm.c, desc))
    with pytest.raises(W.WispError) as e:             # no room for the logits
        W.wisp_verify_kv8(gm.c, kv, desc, t, q, 1, a, o, None, ws)
    assert e.value.status == W.WISP_E_WORKSPACE
    with pytest.raises(ValueError):
        W.wisp_verify_kv8(gm.c, kv.layer(0), desc, t, q, 1, a, o, None, ws)
    logits = torch.empty(3, s.vocab, device="cuda")
    bad = torch.tensor([[0, -1]], dtype=torch.int32, device="cuda")
    W.wisp_verify_kv8(gm.c, kv, W.BatchDesc([20], [2], bad, 1.0), t, q, 1, a, o, logits, ws)
    with pytest.raises(W.WispError) as e:
        W.wisp_check(ws)
    assert e.value.status == W.WISP_E_DEVICE_INPUT
