"""GPU parity of the 8-bit KV cache's operators (wisp_kv8_append, wisp_attention_kv8) against the
fp64 oracle: head layouts and dims, lengths from one token on, pages that end inside a tile, stale
slots and unused pages full of NaN, rows that are not finite, replayed graphs, other streams."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log
from kv8_harness import Case, attention_bound, dev, host_pool, shape
from oracle import kv8

pytestmark = pytest.mark.gpu

#          ctx, rows per request, query heads, kv heads, head_dim, bf16
APPEND = [
    ([0], [1], 4, 4, 64, True),
    ([0], [1], 1, 1, 32, False),
    ([15, 16, 17, 31], [1, 1, 2, 2], 32, 8, 128, True),
    ([5, 0, 1300], [6, 40, 17], 32, 8, 128, True),
    ([13, 2], [19, 1], 64, 8, 128, True),
    ([100, 7], [9, 33], 6, 2, 64, True),
    ([100, 7], [9, 33], 4, 4, 64, False),
    ([3, 60], [30, 5], 6, 3, 96, False),
    ([1, 20], [15, 16], 5, 1, 160, False),
    ([47, 0], [3, 16], 2, 2, 256, False),
    ([9], [100], 3, 1, 224, False),
]


def _append(case, x, pad=0):
    kv = case.pool()
    qkv = torch.zeros(case.M, x.shape[1] + pad, dtype=torch.bfloat16 if case.bf16 else torch.float32, device="cuda")
    qkv.fill_(float("nan"))
    qkv[:, :x.shape[1]] = dev(x, case.bf16)
    q = torch.full((case.M, case.n_q, case.hd), 7.0, dtype=qkv.dtype, device="cuda")
    plan = case.plan()
    W.wisp_kv8_append(plan, kv, qkv[:, :x.shape[1]], q)
    W.wisp_check(plan.ws)
    return kv, q, plan


def _check_append(case, x, kv, q):
    k, v, scale = case.k.copy(), case.v.copy(), case.scale.astype(np.float64)
    wq, wk, wv = kv8.append(k, v, scale, case.pt, case.ctx, case.nrow, x, case.n_q, case.n_kv, case.hd, case.base)
    gk, gv, gs = host_pool(kv)
    # a rotated value: two products and a sum, the table's cosine and sine each rounded once, in fp32
    xs = x.reshape(case.M, -1, case.hd)
    h2 = case.hd // 2
    pair = np.abs(xs[..., :h2]) + np.abs(xs[..., h2:])
    err = 4 * 2.0 ** -24 * np.concatenate([pair, pair], -1)
    tol = err[:, :case.n_q] + (2.0 ** -8 if case.bf16 else 2.0 ** -24) * np.abs(wq)
    assert np.all(np.abs(q.double().cpu().numpy() - wq) <= tol)
    np.testing.assert_array_equal(gs, scale)
    # codes: the oracle's, but where fp32's error reaches a border between two codes
    for g, w, new, sc, order, e in ((gk, k, wk, 0, kv8.k_order(case.hd), err[:, case.n_q:case.n_q + case.n_kv]),
                                    (gv, v, wv, 1, kv8.v_order(case.hd), 0 * wv)):
        written = np.zeros(g.shape, bool)
        r = 0
        for b in range(len(case.ctx)):
            for t in range(int(case.ctx[b]), int(case.ctx[b] + case.nrow[b])):
                blk, s = case.pt[b, t // 16], t % 16
                written[blk][:, order[s]] = True
                got = kv8.VALUES[g[blk][:, order[s]]]
                x_s = new[r] / scale[blk, :, sc][:, None]
                step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(np.abs(x_s), 1e-300))), -6) - 3)
                assert np.all(np.abs(got - x_s) <= 0.5 * step * (1 + 1e-9) + e[r] / scale[blk, :, sc][:, None]), (b, t)
                r += 1
        np.testing.assert_array_equal(g[~written], w[~written])   # old slots rescaled, all else untouched
        assert np.mean(g[written] != w[written]) < 1e-3


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append_matches_oracle(case):
    log(f"append {APPEND[case]}")
    c = Case(*APPEND[case], seed=100 + case)
    x = c.qkv()
    kv, q, plan = _append(c, x, pad=24 if case % 2 else 0)
    _check_append(c, x, kv, q)
    # once more: the same pages
    before = host_pool(kv)
    W.wisp_kv8_append(plan, kv, dev(x, c.bf16), q)
    for a, b in zip(before, host_pool(kv)):
        np.testing.assert_array_equal(a, b)


def test_append_with_scales_that_are_no_powers_of_two():
    c = Case([13, 40, 7], [4, 9, 5], 8, 2, 64, True, seed=9, pow2=False)
    x = c.qkv()
    kv, q, _ = _append(c, x)
    _check_append(c, x, kv, q)


def test_append_of_large_small_and_zero_values():
    """Pages whose values span fp32: scales at the lower end, zeros, and a page whose old slots
    vanish beside a new row that is far larger."""
    c = Case([5, 0, 0, 0], [3, 16, 16, 4], 2, 2, 64, False, seed=11)
    x = c.qkv()
    x[3:19] *= 1e-36
    x[19:35] = 0.0
    x[:3] *= 1e30
    kv, q, _ = _append(c, x.astype(np.float32).astype(np.float64))
    _check_append(c, x.astype(np.float32).astype(np.float64), kv, q)


def test_rows_that_are_not_finite_stay_theirs():
    """A NaN or an infinity in K or V: the rows that attend to it are NaN, the ones before it are
    what they are without it."""
    for where, bad in ((0, np.nan), (1, np.inf), (1, np.nan), (0, -np.inf)):
        c = Case([20, 30], [5, 5], 8, 2, 64, True, seed=21)
        x = c.qkv()
        x[3, (8 + 2 * where) * 64 + 7] = bad          # request 0's fourth row, K or V of kv head 0
        kv, q, plan = _append(c, x)
        ok = np.ones((c.M, c.n_q), bool)
        ok[3:5, :4] = False
        clean = c.queries()
        out = torch.empty(c.M, 8, 64, dtype=torch.bfloat16, device="cuda")
        W.wisp_attention_kv8(plan, kv, dev(clean, True), out)
        got = out.double().cpu().numpy()
        assert np.isnan(got[~ok]).all() and np.isfinite(got[ok]).all()
        k, v, s = host_pool(kv)
        assert not np.isnan(kv8.VALUES[v[c.pt[0, 1]][:, kv8.v_order(64)[:9]]]).any()
        ref, mag, big = kv8.attention(clean, k, v, s, c.pt, c.ctx, c.nrow, 2)
        assert np.all((np.abs(got - ref) <= attention_bound(ref, mag, big, 64, 40, True))[ok])


ATTENTION = [
    ([0], [1], 4, 4, 64, True),
    ([0], [1], 1, 1, 32, False),
    ([0, 1, 15, 16, 31, 32], [1, 1, 1, 1, 1, 1], 32, 8, 128, True),
    ([15, 40, 0, 129], [2, 5, 1, 4], 32, 8, 128, True),
    ([700, 33, 2500], [9, 17, 3], 32, 8, 128, True),
    ([1000, 17], [17, 6], 64, 8, 128, True),
    ([300, 64, 5], [4, 8, 2], 8, 8, 64, True),
    ([64, 900], [3, 10], 16, 2, 64, True),
    ([12000, 900], [7, 4], 32, 8, 128, True),
    ([40, 3], [2, 1], 64, 1, 128, True),         # 64 query heads on one kv head
    ([0, 250], [150, 90], 8, 2, 128, True),      # prompts
    ([513], [3], 6, 2, 64, True),                # three query heads per kv head
    ([700, 33], [9, 17], 8, 2, 128, False),
    ([300, 64, 5], [4, 40, 2], 4, 4, 64, False),
    ([5000], [6], 4, 4, 64, False),
    ([100, 7], [9, 3], 6, 3, 96, False),
    ([31, 200], [4, 17], 5, 1, 160, False),
    ([99], [20], 2, 2, 192, False),
    ([50], [3], 3, 1, 224, False),
    ([47, 330], [3, 16], 2, 2, 256, False),
]


# shapes that reach the plan's corners: many kv heads leave few workgroups for each
PLANS = [
    # long shares: a wave's share is longer than the 64 pages whose ids it holds at a time
    ([5000, 50], [2, 1], 512, 512, 64, True),
    ([5000], [3], 512, 512, 32, False),
    # the same with three row groups, whose waves run alone
    ([9000, 17000], [17, 17], 128, 32, 64, True),
    # many short requests: a workgroup runs one item after another
    ([(37 * k) % 101 for k in range(300)], [1 + k % 5 for k in range(300)], 32, 32, 64, True),
    ([(37 * k) % 101 for k in range(200)], [1 + k % 20 for k in range(200)], 64, 16, 128, True),
    # row groups of 16 rows, all kinds of bundles next to each other
    ([500, 3, 2000, 64, 1], [1, 4, 2, 3, 4], 16, 4, 128, True),
    ([100, 3, 0, 64, 1, 700], [50, 4, 33, 17, 9, 100], 16, 4, 64, True),
    ([100, 3, 0, 64, 1, 700], [50, 4, 33, 17, 9, 100], 16, 4, 64, False),
]


@pytest.mark.parametrize("case", range(len(PLANS)))
def test_attention_at_the_corners_of_the_plan(case):
    ctx, nrow = PLANS[case][:2]
    log(f"attention of {len(ctx)} requests, ctx {min(ctx)}-{max(ctx)}, rows {min(nrow)}-{max(nrow)}, {PLANS[case][2:]}")
    c = Case(*PLANS[case], seed=500 + case, pow2=case % 2 == 1).fill()
    _check_attention(c, c.queries())


def _check_attention(c, q, plan=None, kv=None):
    kv = kv or c.pool()
    plan = plan or c.plan()
    out = torch.full((c.M, c.n_q, c.hd), 7.0, dtype=torch.bfloat16 if c.bf16 else torch.float32, device="cuda")
    W.wisp_attention_kv8(plan, kv, dev(q, c.bf16), out)
    W.wisp_check(plan.ws)
    k, v, s = host_pool(kv)
    ref, mag, big = kv8.attention(q, k, v, s, c.pt, c.ctx, c.nrow, c.n_kv)
    err, tol = np.abs(out.double().cpu().numpy() - ref), attention_bound(ref, mag, big, c.hd, int((c.ctx + c.nrow).max()), c.bf16)
    log(f"  worst {np.max(err / tol):.3f} of its bound, largest error {err.max():.2e}")
    assert np.all(err <= tol)
    return out


@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention_matches_oracle(case):
    log(f"attention {ATTENTION[case]}")
    c = Case(*ATTENTION[case], seed=300 + case, pow2=case % 2 == 0).fill()
    _check_attention(c, c.queries())


# many rows: three and four row groups that run together, apart from the others
WIDE = [
    ([0], [130], 8, 2, 128, True),
    ([3000, 700, 40], [70, 2, 1], 32, 8, 128, True),
    ([5000], [24], 32, 8, 128, True),            # three row groups, cut and joined
    ([64, 1, 333], [33, 64, 65], 16, 2, 64, True),
    ([2000, 9, 0], [40, 300, 16], 8, 4, 64, True),
    ([15, 16, 17], [81, 80, 79], 6, 2, 128, True),
    ([900 + 13 * k for k in range(40)], [25 + k % 9 for k in range(40)], 64, 16, 128, True),   # several for a workgroup
    ([0, 4000], [1000, 1], 4, 1, 128, True),
    ([200, 100, 0], [2, 2, 2], 40, 1, 64, True),  # three row groups of two rows
]


@pytest.mark.parametrize("case", range(len(WIDE)))
def test_attention_of_many_rows(case):
    log(f"attention of {len(WIDE[case][0])} requests, rows {WIDE[case][1][:3]}, {WIDE[case][2:]}")
    c = Case(*WIDE[case], seed=700 + case, pow2=case % 2 == 0).fill()
    _check_attention(c, c.queries())


def test_bad_block_ids_of_many_rows_are_reported():
    c = Case([20], [200], 8, 2, 128, True, seed=43).fill()
    c.pt[0, 7] = c.k.shape[0]
    from gpu_harness import to_dev
    c.desc = W.BatchDesc(c.ctx, c.gamma, to_dev(c.pt), 1.0, None, c.nrow - 1 - c.gamma)
    kv, plan = c.pool(), c.plan()
    q = dev(c.queries(), True)
    W.wisp_attention_kv8(plan, kv, q, torch.empty_like(q))
    with pytest.raises(W.WispError) as e:
        W.wisp_check(plan.ws)
    assert e.value.status == W.WISP_E_DEVICE_INPUT


@pytest.mark.parametrize("n_q,n_kv,hd,lo,hi", [(64, 16, 128, 200, 6000), (16, 16, 128, 1000, 5000), (64, 32, 64, 200, 6000), (32, 32, 64, 10, 6000)])
def test_attention_of_more_codes_than_the_caches_hold(n_q, n_kv, hd, lo, hi):
    _check_large(n_q, n_kv, hd, lo, hi, 1, 18)


@pytest.mark.parametrize("n_q,n_kv,hd,lo,hi", [(64, 16, 128, 200, 6000), (64, 32, 64, 200, 6000)])
def test_attention_of_many_rows_and_more_codes_than_the_caches_hold(n_q, n_kv, hd, lo, hi):
    _check_large(n_q, n_kv, hd, lo, hi, 14, 70)


def _check_large(n_q, n_kv, hd, lo, hi, least, most):
    """Over 256 MB of codes (they are read past the caches then), one to five row groups a request;
    the reference in fp64 on the device."""
    rng = np.random.default_rng(n_q + hd)
    B = 4 + (300 << 20) // (2 * n_kv * hd) // ((lo + hi) // 2)
    ctx, nrow = rng.integers(lo, hi, B).astype(np.int32), rng.integers(least, most, B).astype(np.int32)
    nrow[0] = 40
    tokens = ctx + nrow
    log(f"{B} requests, {int(tokens.sum()) * 2 * n_kv * hd >> 20} MB of codes")
    assert int(tokens.sum()) * 2 * n_kv * hd > 256 << 20
    need = (tokens + 15) // 16
    nb = int(need.sum())
    pt, perm, o = np.full((B, int(need.max())), -1, np.int32), rng.permutation(nb).astype(np.int32), 0
    for b in range(B):
        pt[b, :need[b]] = perm[o:o + need[b]]
        o += need[b]
    g = torch.Generator(device="cuda")
    g.manual_seed(hd)
    pool = lambda: (90.0 * torch.randn(nb, n_kv, 16 * hd, device="cuda", generator=g)).clamp_(-448, 448).to(torch.float8_e4m3fn)
    k, v = pool(), pool()
    scale = torch.exp2(torch.randint(-8, -4, (nb, n_kv, 2), device="cuda", generator=g).float())
    M = int(nrow.sum())
    q = torch.randn(M, n_q, hd, device="cuda", generator=g).to(torch.bfloat16)
    m = W.GpuModel.shape_only(shape(n_q, n_kv, hd, True))
    gamma = np.minimum(nrow - 1, 16)
    desc = W.BatchDesc(ctx, gamma, torch.from_numpy(pt).cuda(), 1.0, None, nrow - 1 - gamma)
    plan = W.wisp_kv8_plan(m, desc, W.workspace(W.wisp_kv8_workspace_size(m, desc)))
    out = torch.empty_like(q)
    W.wisp_attention_kv8(plan, W.KV8Pool(k[None], v[None], scale[None]), q, out)
    W.wisp_check(plan.ws)
    order = [torch.from_numpy(f(hd)).cuda() for f in (kv8.k_order, kv8.v_order)]
    off, G, worst = np.concatenate([[0], np.cumsum(nrow)]), n_q // n_kv, 0.0
    for b in range(B):
        T = int(tokens[b])
        blk = torch.from_numpy(pt[b, :need[b]].astype(np.int64)).cuda()
        kd, vd = [(p[blk].double() * scale[blk][..., w, None].double())[:, :, order[w]].transpose(0, 1).reshape(n_kv, -1, hd)[:, :T]
                  for w, p in enumerate((k, v))]
        qq = q[off[b]:off[b + 1]].double().view(-1, n_kv, G, hd).permute(1, 0, 2, 3).reshape(n_kv, -1, hd)
        s = torch.bmm(qq, kd.transpose(1, 2).contiguous()).view(n_kv, -1, G, T) / hd ** 0.5
        seen = torch.arange(T, device="cuda") <= int(ctx[b]) + torch.arange(int(nrow[b]), device="cuda")[:, None]
        p = torch.softmax(s.masked_fill(~seen[None, :, None], -np.inf), -1).view(n_kv, -1, T)
        ref, mag = torch.bmm(p, vd.contiguous()), torch.bmm(p, vd.abs().contiguous())
        big = torch.bmm(qq.abs(), kd.abs().transpose(1, 2).contiguous()).amax(-1) / hd ** 0.5
        got = out[off[b]:off[b + 1]].double().view(-1, n_kv, G, hd).permute(1, 0, 2, 3).reshape(n_kv, -1, hd)
        tol = attention_bound(*[t.cpu().numpy() for t in (ref, mag, big)], hd, T, True)
        ratio = np.abs((got - ref).cpu().numpy()) / tol
        worst = max(worst, ratio.max())
        assert worst <= 1.0, (b, worst)
    log(f"  worst {worst:.3f} of its bound")


def test_attention_of_peaked_scores():
    """Scores of hundreds: the running maximum rises over and over, probabilities vanish."""
    for bf16 in (True, False):
        c = Case([1500, 3], [5, 3], 8, 2, 64, bf16, seed=77).fill()
        _check_attention(c, c.queries(std=60.0))


@pytest.mark.parametrize("bf16", [True, False])
def test_append_then_attention(bf16):
    """The two as a layer runs them, over three steps of drafts of which some are kept."""
    c = Case([20, 0, 333], [6, 3, 10], 8, 2, 64, bf16, seed=31)
    kv = c.pool()
    host = [c.k.copy(), c.v.copy(), c.scale.astype(np.float64)]
    kept = [[2, 3, 1], [1, 1, 1], [4, 2, 1]]
    rng = np.random.default_rng(8)
    for step, keep in enumerate(kept):
        x = c.qkv()
        plan = c.plan()
        q = torch.empty(c.M, 8, 64, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda")
        W.wisp_kv8_append(plan, kv, dev(x, bf16), q)
        qh = q.double().cpu().numpy()
        _check_attention(c, qh, plan, kv)
        kv8.append(*host, c.pt, c.ctx, c.nrow, x, 8, 2, 64, c.base)
        np.testing.assert_array_equal(host_pool(kv)[2], host[2])
        c.ctx = c.ctx + np.asarray(keep, np.int32)        # rollback by length
        c.nrow = rng.integers(1, 8, 3).astype(np.int32)
        need = (c.ctx + c.nrow + 15) // 16
        for b in range(3):                                # pages that the longer requests need
            while (c.pt[b] >= 0).sum() < need[b]:
                c.pt[b, (c.pt[b] >= 0).sum()] = max(set(range(c.k.shape[0])) - set(c.pt.reshape(-1).tolist()))
        c.M = int(c.nrow.sum())
        from gpu_harness import to_dev
        c.desc = W.BatchDesc(c.ctx, c.nrow - 1, to_dev(c.pt), 1.0)


def test_bad_block_ids_are_reported():
    c = Case([40, 20], [3, 3], 8, 2, 64, True, seed=41).fill()
    for bad in (-1, c.k.shape[0], 1 << 30):
        keep = c.pt[0, 2]
        c.pt[0, 2] = bad
        from gpu_harness import to_dev
        c.desc = W.BatchDesc(c.ctx, c.nrow - 1, to_dev(c.pt), 1.0)
        kv, plan = c.pool(), c.plan()
        before = host_pool(kv)
        q = torch.empty(c.M, 8, 64, dtype=torch.bfloat16, device="cuda")
        W.wisp_kv8_append(plan, kv, dev(c.qkv(), True), q)
        with pytest.raises(W.WispError) as e:
            W.wisp_check(plan.ws)
        assert e.value.status == W.WISP_E_DEVICE_INPUT
        W.wisp_attention_kv8(plan, kv, q, torch.empty_like(q))
        with pytest.raises(W.WispError):
            W.wisp_check(plan.ws)
        W.wisp_check(plan.ws)                            # cleared
        touched = {int(c.pt[0, 2]), int(c.pt[1, 1])}
        for a, b in zip(before, host_pool(kv)):
            for blk in range(a.shape[0]):
                if blk not in touched:
                    np.testing.assert_array_equal(a[blk], b[blk])
        c.pt[0, 2] = keep


def test_captured_and_replayed():
    """Append and attention in a graph, replayed with new inputs between eager calls; a plan made
    while capturing."""
    c = Case([900, 33], [6, 3], 32, 8, 128, True, seed=51)
    kv, plan = c.pool(), c.plan()
    qkv = dev(c.qkv(), True)
    q = torch.empty(c.M, 32, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    side = torch.cuda.Stream()
    ws = W.workspace(W.wisp_kv8_workspace_size(c.model, c.desc))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        inner = W.wisp_kv8_plan(c.model, c.desc, ws)
        W.wisp_kv8_append(inner, kv, qkv, q)
        W.wisp_attention_kv8(inner, kv, q, out)
    for step in range(4):
        qkv.copy_(dev(c.qkv(), True))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        W.wisp_check(ws)
        kv2, q2 = c.pool(), torch.empty_like(q)
        out2 = torch.empty_like(q)
        W.wisp_kv8_append(plan, kv2, qkv, q2)
        W.wisp_attention_kv8(plan, kv2, q2, out2)
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and torch.equal(out, out2), step


def test_two_plans_on_two_streams():
    c = [Case([900, 33], [6, 3], 32, 8, 128, True, seed=61 + k).fill() for k in range(2)]
    q = [dev(x.queries(), True) for x in c]
    kv = [x.pool() for x in c]
    plans = [x.plan() for x in c]
    alone = []
    for p, k, x in zip(plans, kv, q):
        alone.append(torch.empty_like(x))
        W.wisp_attention_kv8(p, k, x, alone[-1])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in c]
    outs = [torch.empty_like(x) for x in q]
    for _ in range(20):
        for p, k, x, o, s in zip(plans, kv, q, outs, streams):
            W.wisp_attention_kv8(p, k, x, o, s)
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)


def test_pages_beyond_4_gib_of_pool():
    """The same batch in a small pool and at the end of one of 4.6 GB: the same results, bit for bit."""
    from gpu_harness import to_dev
    c = Case([900, 0, 33], [6, 150, 3], 32, 8, 128, True, seed=91)
    nb, n_big = c.k.shape[0], 280000
    assert n_big * 8 * 2048 > 1 << 32
    small, big = c.pool(), W.KV8Pool.zeros(1, n_big, 8, 128)
    for b, a in ((big.k, small.k), (big.v, small.v)):
        b.view(torch.uint8)[0, n_big - nb:] = a.view(torch.uint8)[0]
    big.scale[0, n_big - nb:] = small.scale[0]
    x = dev(c.qkv(), True)
    out = []
    for kv, shift in ((small, 0), (big, n_big - nb)):
        pt = np.where(c.pt >= 0, c.pt + shift, -1).astype(np.int32)
        d = W.BatchDesc(c.ctx, c.gamma, to_dev(pt), 1.0, None, c.nrow - 1 - c.gamma)
        plan = W.wisp_kv8_plan(c.model, d, W.workspace(W.wisp_kv8_workspace_size(c.model, d)))
        q = torch.empty(c.M, 32, 128, dtype=torch.bfloat16, device="cuda")
        o = torch.empty_like(q)
        W.wisp_kv8_append(plan, kv, x, q)
        W.wisp_attention_kv8(plan, kv, q, o)
        W.wisp_check(plan.ws)
        out.append((q, o, kv.k.view(torch.uint8)[0, shift:shift + nb], kv.v.view(torch.uint8)[0, shift:shift + nb]))
    for a, b in zip(*out):
        assert torch.equal(a, b)
    assert int(big.k.view(torch.uint8)[0, :nb].max()) == 0


def test_wrapper_refuses_tensors_that_do_not_fit():
    c = Case([40, 20], [3, 3], 8, 2, 64, True, seed=71).fill()
    kv, plan = c.pool(), c.plan()
    q = torch.empty(c.M, 8, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(c.M, 12 * 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: W.wisp_attention_kv8(plan, kv, q.float(), q),
                 lambda: W.wisp_attention_kv8(plan, kv, q[1:], q),
                 lambda: W.wisp_attention_kv8(plan, kv, q.cpu(), q),
                 lambda: W.wisp_attention_kv8(plan, kv, q.transpose(1, 2), q),
                 lambda: W.wisp_kv8_append(plan, kv, x[:, 1:], q),
                 lambda: W.wisp_kv8_append(plan, kv, x[1:], q),
                 lambda: W.wisp_kv8_append(plan, W.KV8Pool.zeros(1, 4, 2, 128), x, q),
                 lambda: W.KV8Pool(kv.k, kv.v, kv.scale[..., 0]),
                 lambda: W.KV8Pool(kv.k.view(torch.uint8), kv.v, kv.scale)):
        with pytest.raises(ValueError):
            call()
    wide = torch.zeros(c.M, 12 * 64 + 8, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(W.WispError):                      # rows not 16-byte aligned
        W.wisp_kv8_append(plan, kv, wide[:, 4:4 + 12 * 64], q)
    with pytest.raises(W.WispError):
        W.wisp_kv8_append(plan, kv, x[:1].expand(c.M, -1), q)
    with pytest.raises(W.WispError):
        W.wisp_kv8_plan(c.model, c.desc, W.workspace(256))
    W.wisp_attention_kv8(plan, kv, q, torch.empty_like(q))
    W.wisp_check(plan.ws)


def test_an_empty_batch_does_nothing():
    m = Case([3], [1], 8, 2, 64, True, seed=1).model
    d = W.BatchDesc([], [], torch.zeros(0, 1, dtype=torch.int32, device="cuda"), 1.0)
    plan = W.wisp_kv8_plan(m, d, W.workspace(256))
    e = torch.empty(0, 8, 64, dtype=torch.bfloat16, device="cuda")
    W.wisp_attention_kv8(plan, W.KV8Pool.zeros(1, 2, 2, 64), e, e)
    W.wisp_kv8_append(plan, W.KV8Pool.zeros(1, 2, 2, 64), torch.empty(0, 12 * 64, dtype=torch.bfloat16, device="cuda"), e)
