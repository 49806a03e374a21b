"""GPU parity of wisp_token_logprobs against fp64: vocabularies from one entry on, rows at any
alignment, masks (-infinity, the type's lowest value, all of a row), equal values, NaN and +infinity,
rows without a token, replayed graphs."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log


def _ref(x, T, tok, top):
    """fp64 (lp, H, ids, tlp) of one row and what fp32's exponentials and sums may add to lp and H:
    each exponential is off by 2^-22 of its exponent (two roundings of it) and 2^-23, a sum by
    at most 45 half steps."""
    z = x.astype(np.float64) / T
    fin, d = np.isfinite(z), z
    if np.isnan(z).any() or (z == np.inf).any():
        lp = H = ls = np.nan
        b1 = b2 = 0.0
    elif not fin.any():
        ls, H, b1, b2 = -np.inf, 0.0, 0.0, 0.0
        lp = -np.inf
    else:
        d = z - z[fin].max()                # before anything is added: 3.4e38 would swallow it
        e = np.where(fin, np.exp(np.where(fin, d, 0.0)), 0.0)
        p, dd = e / e.sum(), np.where(fin, d, 0.0)
        ls = np.log(e.sum())
        lp = d[tok] - ls if tok is not None else np.nan
        H = ls - (p * dd).sum()
        s1, s2 = (p * -dd).sum(), (p * dd * dd).sum()
        b1 = 2.0 ** -22 * (s1 + 16)
        b2 = b1 + 2.0 ** -22 * (s2 + 16 * s1)
    order = np.lexsort((np.arange(x.size), -np.where(np.isnan(x), -np.inf, x)))
    order = order[(x[order] > -np.inf) & ~np.isnan(x[order])][:top]
    ids = np.full(top, -1)
    tlp = np.full(top, np.nan if np.isnan(ls) else -np.inf)
    ids[:order.size] = order
    tlp[:order.size] = np.nan if np.isnan(ls) else d[order] - ls
    return lp, H, ids, tlp, b1, b2


def _check(x, V, tok, T, top, got, rows=None):
    lp, H, ids, tlp = [None if g is None else g.double().cpu().numpy() for g in got]
    xs = x[:, :V].float().cpu().numpy()
    worst = 0.0
    for r in range(xs.shape[0]) if rows is None else rows:
        t = None if tok is None else int(tok[r])
        a, h, wi, wl, b1, b2 = _ref(xs[r], T, t, top)
        for g, w, b in ((lp[r] if lp is not None else None, a, b1), (H[r] if H is not None else None, h, b2)):
            if g is None:
                continue
            if not np.isfinite(w):
                assert (np.isnan(g) and np.isnan(w)) or g == w, (r, g, w)
            else:
                tol = 2.0 ** -23 * abs(w) + b
                worst = max(worst, abs(g - w) / max(tol, 1e-30))
                assert abs(g - w) <= tol, (r, g, w)
        if top:
            np.testing.assert_array_equal(ids[r], wi)
            fin = np.isfinite(wl)
            assert np.array_equal(np.isnan(tlp[r]), np.isnan(wl)) and np.all(tlp[r][~fin & ~np.isnan(wl)] == -np.inf)
            assert np.all(np.abs(tlp[r][fin] - wl[fin]) <= 2.0 ** -23 * np.abs(wl[fin]) + b1)
    return worst


def _run(x, V, tok, T, top, stream=None):
    rows = x.shape[0]
    lp = torch.full((rows,), 7.0, device="cuda") if tok is not None else None
    H = torch.full((rows,), 7.0, device="cuda")
    ids = torch.full((rows, top), 7, dtype=torch.int32, device="cuda") if top else None
    tlp = torch.full((rows, top), 7.0, device="cuda") if top else None
    ws = W.workspace(W.wisp_token_logprobs_workspace_size(rows, V, top))
    W.wisp_token_logprobs(x, V, tok, T, lp, H, ids, tlp, ws, stream)
    return (lp, H, ids, tlp), ws


def _logits(rows, V, dtype, seed, pad=0, shift=0, std=2.5):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n = V + pad
    flat = torch.full((rows * n + shift,), float("nan"), dtype=dtype, device="cuda")
    x = flat[shift:].view(rows, n)
    x[:, :V] = (std * torch.randn(rows, V, device="cuda", generator=g)).to(dtype)
    tok = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32, generator=g)
    return x, tok


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top,pad,shift,T", [
    (1, 1, 1, 0, 0, 1.0), (3, 5, 8, 0, 0, 1.0), (2, 63, 20, 1, 0, 0.5), (4, 500, 5, 12, 1, 1.0), (5, 8192, 20, 0, 0, 1.0),
    (3, 8193, 32, 7, 0, 2.0), (2, 8191, 0, 8, 8, 1.0), (7, 50021, 8, 27, 0, 0.7), (9, 128256, 20, 0, 0, 1.0),
    (2, 200001, 32, 3, 3, 1.0), (65, 1000, 3, 0, 0, 0.05), (2, 128256, 1, 0, 0, 30.0),
])
def test_matches_fp64(rows, V, top, pad, shift, T, dtype):
    log(f"logprobs rows={rows} V={V} top={top} pad={pad} shift={shift} T={T} {dtype}")
    x, tok = _logits(rows, V, dtype, 7 * V + rows, pad, shift)
    got, ws = _run(x, V, tok, T, top)
    W.wisp_check(ws)
    log(f"  worst {_check(x, V, tok, T, top, got):.3f} of its bound")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 20000, 128256])
def test_masks_equal_values_and_orders(V, dtype):
    x, tok = _logits(13, V, dtype, V)
    low = torch.finfo(dtype).min
    x[0] = -float("inf")                       # nothing left
    x[1] = -float("inf")
    x[1, V // 2] = 3.0                         # one token left
    x[2] = low                                 # the lowest value as a mask: three left
    x[2, [V // 3, 5, V - 1]] = torch.tensor([1.0, 1.0, -2.0], device="cuda", dtype=dtype)
    x[3] = 0.0                                 # all equal
    x[4] = low
    x[5] = torch.arange(V, device="cuda").to(dtype) * 1e-3
    x[6] = -torch.arange(V, device="cuda").to(dtype) * 1e-3
    x[7, ::3] = -float("inf")
    x[8, 100:] = -float("inf")                 # fewer than a wave's
    x[9] = (x[9] > 0).to(dtype)                # two values
    x[10] += 20000.0                           # a large offset
    x[11, V // 2:] = 50.0                      # half of them the largest
    x[12, :V - 40] = 0.0                       # equal, the others anywhere around
    tok[1], tok[2], tok[8] = V // 2, 5, 3
    for top in (0, 1, 20, 32):
        got, ws = _run(x, V, tok, 1.0, top)
        W.wisp_check(ws)
        log(f"  V={V} top={top}: worst {_check(x, V, tok, 1.0, top, got):.3f} of its bound")


@pytest.mark.gpu
def test_values_that_are_not_finite():
    x, tok = _logits(4, 9000, torch.float32, 3)
    x[0, 77] = float("nan")
    x[1, 8999] = float("inf")
    x[2] = float("nan")
    tok[3] = 4
    x[3, 4] = -float("inf")                    # the token itself is masked
    got, _ = _run(x, 9000, tok, 1.0, 5)
    _check(x, 9000, tok, 1.0, 5, got, rows=[0, 2, 3])
    lp, H, ids, tlp = got
    assert torch.isnan(lp[1]) and torch.isnan(H[1]) and torch.isnan(tlp[1]).all() and int(ids[1, 0]) == 8999


@pytest.mark.gpu
@pytest.mark.parametrize("V", [40, 5000, 90000])
def test_zeros_of_either_sign_are_equal(V):
    x, tok = _logits(3, V, torch.float32, V)
    x[0] = -x[0].abs()
    x[0, ::7], x[0, 3::7] = -0.0, 0.0          # the largest: by index, whichever sign
    x[1] = 0.0
    x[1, ::2] = -0.0
    x[2] = -x[2].abs()
    x[2, V - 3:], x[2, 2] = 0.0, -0.0          # a few
    for top in (1, 6, 32):
        got, _ = _run(x, V, tok, 1.0, top)
        _check(x, V, tok, 1.0, top, got)


@pytest.mark.gpu
def test_rows_without_a_token_are_left():
    x, tok = _logits(6, 30000, torch.float32, 5)
    tok[[0, 3, 5]] = -1
    got, ws = _run(x, 30000, tok, 1.0, 4)
    W.wisp_check(ws)
    _check(x, 30000, tok, 1.0, 4, got, rows=[1, 2, 4])
    for g in got:
        assert (g[[0, 3, 5]] == 7).all()
    # no tokens at all: every row's entropy and top tokens
    got, _ = _run(x, 30000, None, 1.0, 4)
    _check(x, 30000, None, 1.0, 4, got)


@pytest.mark.gpu
def test_tokens_out_of_range_are_reported():
    x, tok = _logits(3, 1000, torch.float32, 6)
    for bad in (1000, -2, 2 ** 31 - 1):
        tok[1] = bad
        got, ws = _run(x, 1000, tok, 1.0, 2)
        with pytest.raises(W.WispError) as e:
            W.wisp_check(ws)
        assert e.value.status == W.WISP_E_DEVICE_INPUT
        assert torch.isnan(got[0][1])
        _check(x, 1000, tok, 1.0, 2, got, rows=[0, 2])


@pytest.mark.gpu
def test_more_rows_than_a_launch_has_threads_for():
    rows, V = (1 << 24) + 4097, 3
    x, tok = _logits(rows, V, torch.float32, 9)
    tok[5::2] = -1
    (lp, H, _, _), ws = _run(x, V, tok, 1.0, 0)
    W.wisp_check(ws)
    log(f"logprobs of {rows} rows")
    keep = tok != -1
    ls = torch.log_softmax(x.double(), -1)
    want = ls.gather(1, tok.clamp_min(0).long()[:, None])[:, 0]
    # three entries: each sum takes a handful of fp32 roundings of terms below 16
    assert ((lp.double() - want).abs()[keep] <= 64 * 2.0 ** -24 * (1 + want.abs()[keep])).all()
    assert ((H.double() + (ls.exp() * ls).sum(-1)).abs()[keep] <= 64 * 2.0 ** -24 * 16).all()
    assert (lp[~keep] == 7).all() and (H[~keep] == 7).all()


@pytest.mark.gpu
def test_logits_beyond_2_31_entries():
    """The last rows of 8.6 GB of logits: as by themselves, bit for bit."""
    rows, V, k = 16900, 128256, 3
    assert (rows - k) * V > 1 << 31
    x = torch.zeros(rows, V, device="cuda")
    tail, tok = _logits(k, V, torch.float32, 12)
    x[-k:] = tail
    all_tok = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    all_tok[-k:] = tok
    got, ws = _run(x, V, all_tok, 1.0, 5)
    W.wisp_check(ws)
    alone, _ = _run(tail, V, tok, 1.0, 5)
    for a, b in zip(got, alone):
        assert torch.equal(a[-k:], b) and (a[:-k] == 7).all()


@pytest.mark.gpu
def test_captured_replayed_and_on_two_streams():
    x, tok = _logits(20, 40000, torch.float32, 8)
    rows, V, top = 20, 40000, 6
    outs = lambda: (torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"),
                    torch.zeros(rows, top, dtype=torch.int32, device="cuda"), torch.zeros(rows, top, device="cuda"))
    a, b = outs(), outs()
    ws = [W.workspace(W.wisp_token_logprobs_workspace_size(rows, V, top)) for _ in range(2)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        W.wisp_token_logprobs(x, V, tok, 1.0, *a, ws[0])
    for step in range(4):
        x.copy_(_logits(rows, V, torch.float32, 80 + step)[0])
        torch.cuda.synchronize()
        graph.replay()
        W.wisp_token_logprobs(x, V, tok, 1.0, *b, ws[1], torch.cuda.Stream())
        torch.cuda.synchronize()
        for p, q in zip(a, b):
            assert torch.equal(p, q)
        _check(x, V, tok, 1.0, top, a)


def test_refusals():
    L, FAKE = W.load_library(), 0x1000
    f = lambda dtype=0, rows=2, V=100, ld=100, T=1.0, tok=FAKE, top=2, lp=FAKE, ids=FAKE, tlp=FAKE, ws=FAKE, n=1 << 40, x=FAKE: \
        L.wisp_token_logprobs(x, dtype, rows, V, ld, C.c_float(T), tok, top, lp, FAKE, ids, tlp, ws, n, None)
    for kw in (dict(rows=-1), dict(V=0), dict(ld=99), dict(T=0.0), dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan")),
               dict(top=-1), dict(top=33), dict(tok=None), dict(ids=None), dict(tlp=None), dict(ws=None), dict(x=None),
               dict(ws=FAKE + 4), dict(x=FAKE + 2)):
        assert f(**kw) == W.WISP_E_INVALID, kw
    assert f(dtype=2) == W.WISP_E_UNSUPPORTED
    assert f(V=(1 << 30) + 1, ld=1 << 31) == W.WISP_E_UNSUPPORTED
    assert f(rows=1 << 30, V=100000, ld=100000) == W.WISP_E_UNSUPPORTED
    assert f(n=256) == W.WISP_E_WORKSPACE
    assert f(rows=0) == W.WISP_OK
    assert W.wisp_token_logprobs_workspace_size(2, 100, 33) == 0
    assert W.wisp_token_logprobs_workspace_size(2, 100, 0) < W.wisp_token_logprobs_workspace_size(2, 100, 1)
