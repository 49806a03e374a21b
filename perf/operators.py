"""Measured cases of the operators around an 8-bit KV cache, through the library's public entry
points and in their plain form:

  wisp_kv8_append       rotates the new rows' Q and K by their positions and appends K and V to a
                        paged cache of e4m3 codes with one scale for each page and kv head
  wisp_attention_kv8    one layer's ragged paged attention over that cache
  wisp_token_logprobs   log probabilities of given tokens, entropy and the most probable tokens

The plain form is written in elementary torch operations in fp32 (angles in fp64), over batches
padded to their longest request; `exact` states the same operators in fp64, request by request.
A cache is returned as the e4m3 values and the scales that it holds.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
E4M3_MAX = 448.0
# query heads, kv heads, head_dim, storage, rotary base: the heads of the served model shapes
SHAPES = {
    "tiny": (4, 4, 64, "f32", 1e4),
    "8b": (32, 8, 128, "bf16", 5e5),
    "70b": (64, 8, 128, "bf16", 5e5),
}
STD = 1.15             # of rotated heads: what projections of unit-RMS rows give


class Heads:
    def __init__(self, key):
        self.nq, self.nkv, self.hd, self.dtype, self.base = SHAPES[key]
        self.name, self.group = key, self.nq // self.nkv
        self.torch = torch.float32 if self.dtype == "f32" else torch.bfloat16
        self.es = 4 if self.dtype == "f32" else 2
        # what the library's model descriptor holds besides: not read by these operators
        self.n_layers, self.d_model, self.n_q_heads, self.n_kv_heads = 1, self.nq * self.hd, self.nq, self.nkv
        self.head_dim, self.d_ff, self.vocab, self.rms_eps, self.rope_base = self.hd, self.nq * self.hd, 1024, 1e-5, self.base


# ------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------
def _batch(name, kind, shape, requests, ctx, gamma, cold=0, prompt=(0, 0), plain=0.0, mix=1, pad=0):
    """`cold` first-time requests (prompts of `prompt` rows, log-uniform) before `requests`
    follow-ups of ctx cached tokens (log-uniform), each with gamma drafts (a share `plain` of
    them with none); pad: elements between the rows of the projection's output."""
    return dict(name=name, kind=kind, shape=shape, requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1], gamma_lo=gamma[0],
                gamma_hi=gamma[1], plain=plain, cold=cold, prompt_lo=prompt[0], prompt_hi=prompt[1], mix=mix, pad=pad)


def _logprobs(name, rows, vocab, top, dtype="f32", share=1.0, temperature=1.0, pad=0, mix=1):
    return dict(name=name, kind="logprobs", rows=rows, vocab=vocab, top=top, dtype=dtype, share=share,
                temperature=temperature, pad=pad, mix=mix)


def listed():
    return [
        # one session in a chat, a layer's append: the least that a server does at a time
        _batch("append_8b_b1", "append", "8b", 1, (1300, 1300), (5, 5)),
        # the same for 32 sessions of 512-2048 cached tokens
        _batch("append_8b_b32", "append", "8b", 32, (512, 2048), (1, 8), mix=18),
        # first verifications of long prompts among running sessions
        _batch("append_8b_prefill", "append", "8b", 10, (128, 2048), (1, 8), cold=6, prompt=(1000, 4000), mix=3),
        # a small fp32 model, its rows inside a wider buffer, some requests new
        _batch("append_tiny_f32", "append", "tiny", 16, (1, 500), (0, 16), cold=2, prompt=(5, 60), mix=5, pad=64),
        # one layer's attention of one session
        _batch("attention_8b_b1", "attention", "8b", 1, (1300, 1300), (5, 5)),
        # of 32 sessions
        _batch("attention_8b_b32", "attention", "8b", 32, (512, 2048), (1, 8), mix=18),
        # of 128 sessions with contexts of very different lengths, a quarter plain decoding
        _batch("attention_8b_dyn128", "attention", "8b", 128, (256, 32768), (1, 16), plain=0.25),
        # of a long prompt's first verification with one short follow-up caught in its batch
        _batch("attention_8b_prefill", "attention", "8b", 1, (500, 500), (5, 5), cold=1, prompt=(4096, 4096)),
        # of a small fp32 model's sessions
        _batch("attention_tiny_f32", "attention", "tiny", 24, (64, 4096), (0, 8), mix=4),
        # what one session's answer says about its tokens
        _logprobs("logprobs_b1", 6, 128256, 5),
        # the same of 256 sessions; rows past the accepted drafts have no token
        _logprobs("logprobs_b256", 1237, 128256, 20, share=0.6),
        # bf16 logits (many equal values) of an odd vocabulary in padded rows
        _logprobs("logprobs_bf16_odd", 300, 50021, 8, dtype="bf16", temperature=0.7, pad=27),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(["append", "attention", "prefill", "logprobs"], [3, 4, 2, 3])[0]
    mix = rng.randrange(1, 1 << 30)
    if kind == "logprobs":
        vocab = _log_int(rng, 500, 200000)
        return {k: v for k, v in _logprobs("", _log_int(rng, 1, max(1, min(4096, 1237 * 128256 // vocab))), vocab, rng.randint(0, 20),
                                           dtype=rng.choice(["f32", "f32", "bf16"]), share=rng.choice([1.0, rng.uniform(0.2, 1.0)]),
                                           temperature=rng.choice([1.0, rng.uniform(0.3, 2.0)]), pad=rng.randint(0, 40), mix=mix).items() if k != "name"}
    shape = rng.choices(["8b", "70b", "tiny"], [5, 3, 2])[0]
    if kind == "attention":
        n = _log_int(rng, 1, 256)
        hi = _log_int(rng, 256, min(32768, (800 if shape != "70b" else 400) * 1024 // n))
        g_hi = rng.randint(0, 16 if n < 64 else 8)
        c = _batch("", "attention", shape, n, (max(1, int(hi * rng.uniform(0.02, 1.0))), hi), (rng.randint(0, g_hi), g_hi),
                   plain=rng.choice([0.0, 0.25]), mix=mix)
    elif kind == "append":
        n = _log_int(rng, 1, 256)
        hi = _log_int(rng, 16, 2048)
        g_hi = rng.randint(0, 16)
        c = _batch("", "append", shape, n, (max(1, int(hi * rng.uniform(0.02, 1.0))), hi), (rng.randint(0, g_hi), g_hi),
                   plain=rng.choice([0.0, 0.25]), mix=mix, pad=8 * rng.randint(0, 16))
    else:
        cold = rng.randint(1, 4)
        hi = _log_int(rng, 40, 4000 // cold)
        c = _batch("", rng.choice(["append", "attention"]), "8b" if shape == "70b" else shape, rng.randint(0, 12),
                   (16, _log_int(rng, 32, 2000)), (0, rng.randint(1, 8)), cold=cold,
                   prompt=(max(1, int(hi * rng.uniform(0.1, 1.0))), hi), mix=mix)
    return {k: v for k, v in c.items() if k != "name"}


def _lengths(case):
    """(cached tokens, prompt rows, drafts) of each request, from the case alone."""
    r = np.random.default_rng([case["mix"], 811])

    def log_ints(lo, hi, n):
        return np.clip(np.rint(np.exp(r.uniform(math.log(lo), math.log(hi), n))), lo, hi).astype(np.int32)

    n, cold = case["requests"], case["cold"]
    gam = r.integers(case["gamma_lo"], case["gamma_hi"], n + cold, endpoint=True).astype(np.int32)
    gam = np.where(r.random(n + cold) < case["plain"], 0, gam).astype(np.int32)
    ctx, pre = np.zeros(n + cold, np.int32), np.zeros(n + cold, np.int32)
    ctx[cold:] = log_ints(case["ctx_lo"], case["ctx_hi"], n)
    if cold:
        pre[:cold] = log_ints(case["prompt_lo"], case["prompt_hi"], cold)
    return ctx, pre, gam


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) & ((1 << 62) - 1))
    return g


def _normal(shape, std, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _page_table(tokens, seed):
    """Scattered pages: a permutation of the pool, -1 past a request's last page."""
    need = (tokens.astype(np.int64) + PAGE - 1) // PAGE
    n_blocks = int(need.sum()) + 3
    perm = np.random.default_rng([int(seed), 7]).permutation(n_blocks).astype(np.int32)
    tab = np.full((len(need), int(need.max())), -1, np.int32)
    o = 0
    for i, k in enumerate(need):
        tab[i, :k] = perm[o:o + k]
        o += k
    return tab, n_blocks


def _pool(h, n_blocks, g):
    """e4m3 pages [n_blocks][n_kv][16 * hd] whose largest values use the type's range."""
    x = torch.empty(n_blocks, h.nkv, PAGE * h.hd, dtype=torch.float8_e4m3fn, device="cuda")
    for a in range(0, n_blocks, 8192):
        b = min(n_blocks, a + 8192)
        x[a:b] = _normal((b - a, h.nkv, PAGE * h.hd), 90.0, torch.float32, g).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return x


def _k_order(hd):
    """[16][hd] -> place of (slot, dim) in a K page."""
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return (((e // 32) * 4 + (e % 32) // 8) * 8 + (s // 8) * 4 + s % 4) * 16 + ((s // 4) % 2) * 8 + e % 8


def _v_order(hd):
    """[16][hd] -> place of (slot, dim) in a V page."""
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return ((e // 32) * 2 + s // 8) * 256 + (e % 16) * 16 + ((e // 16) % 2) * 8 + s % 8


def _ints(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int64), device="cuda")


def prepare(case, seed):
    if case["kind"] == "logprobs":
        return _prepare_logprobs(case, seed)
    h = Heads(case["shape"])
    ctx, pre, gam = _lengths(case)
    nrow = pre + gam + 1
    tab, n_blocks = _page_table(ctx + nrow, seed)
    off = np.concatenate([[0], np.cumsum(nrow)])
    M = int(off[-1])
    req = np.repeat(np.arange(len(ctx)), nrow)
    pos = ctx[req] + np.arange(M) - off[req]
    g = _gen(seed, 2)
    st = dict(kind=case["kind"], h=h, k=_pool(h, n_blocks, g), v=_pool(h, n_blocks, g), M=M, n=len(ctx),
              scale=torch.exp2(torch.randint(-8, -4, (n_blocks, h.nkv, 2), device="cuda", generator=g).float()),
              pt=torch.as_tensor(tab, device="cuda"), ctx=_ints(ctx), off=_ints(off), nrow=_ints(nrow), req=_ints(req),
              pos=_ints(pos), row=_ints(np.arange(M) - off[req]), most_rows=int(nrow.max()), most_tokens=int((ctx + nrow).max()),
              k_order=_ints(_k_order(h.hd)), v_order=_ints(_v_order(h.hd)))
    if case["kind"] == "append":
        N = (h.nq + 2 * h.nkv) * h.hd
        st["qkv"] = _normal((M, N + case["pad"]), STD, h.torch, _gen(seed, 3))[:, :N]
        st["q"] = torch.empty(M, h.nq, h.hd, dtype=h.torch, device="cuda")
        # the pages that get new rows: request, place in its table, valid slots before and after
        first, last = ctx // PAGE, (ctx + nrow - 1) // PAGE
        unit0 = np.concatenate([[0], np.cumsum(last - first + 1)])
        ureq = np.repeat(np.arange(len(ctx)), last - first + 1)
        upage = first[ureq] + np.arange(unit0[-1]) - unit0[ureq]
        st.update(ublk=_ints(tab[ureq, upage]), held=_ints(np.clip(ctx[ureq] - upage * PAGE, 0, PAGE)),
                  filled=_ints(np.clip((ctx + nrow)[ureq] - upage * PAGE, 0, PAGE)), unit=_ints(unit0[req] + pos // PAGE - first[req]))
    else:
        st["q"] = _normal((M, h.nq, h.hd), STD, h.torch, _gen(seed, 3))
        st["out"] = torch.empty_like(st["q"])
    if own:
        import paper_2601_11652_amd as W
        model = W.GpuModel.shape_only(h)
        desc = W.BatchDesc(ctx, gam, st["pt"], 1.0, None, pre if pre.any() else None)
        st["kv"] = W.KV8Pool(st["k"][None], st["v"][None], st["scale"][None])
        st["plan"] = W.wisp_kv8_plan(model, desc, W.workspace(W.wisp_kv8_workspace_size(model, desc)))
    return st


def _prepare_logprobs(case, seed):
    g = _gen(seed, 5)
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    x = _normal((rows, vocab + case["pad"]), 2.5, dt, g)[:, :vocab]
    tok = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32, generator=g)
    keep = np.random.default_rng([case["mix"], 31]).random(rows) < case["share"]   # from the case: its work is known
    keep[0] = True
    tok = torch.where(torch.as_tensor(keep, device="cuda"), tok, -1)
    st = dict(kind="logprobs", x=x, tok=tok, top=min(top, vocab), T=case["temperature"], vocab=vocab,
              lp=torch.zeros(rows, device="cuda"), H=torch.zeros(rows, device="cuda"))
    st["ids"] = torch.full((rows, top), -1, dtype=torch.int32, device="cuda") if top else None
    st["tlp"] = torch.zeros(rows, top, device="cuda") if top else None
    if own:
        import paper_2601_11652_amd as W
        st["ws"] = W.workspace(W.wisp_token_logprobs_workspace_size(rows, vocab, top))
    return st


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(st):
    if st["kind"] == "append":
        if own:
            import paper_2601_11652_amd as W
            W.wisp_kv8_append(st["plan"], st["kv"], st["qkv"], st["q"])
        else:
            _append(st)
        return {"q": st["q"], "k": st["k"], "v": st["v"], "scale": st["scale"]}
    if st["kind"] == "attention":
        if own:
            import paper_2601_11652_amd as W
            W.wisp_attention_kv8(st["plan"], st["kv"], st["q"], st["out"])
            return st["out"]
        return _attention(st)
    if own:
        import paper_2601_11652_amd as W
        W.wisp_token_logprobs(st["x"], st["vocab"], st["tok"], st["T"], st["lp"], st["H"], st["ids"], st["tlp"], st["ws"])
        return {k: st[k] for k in ("lp", "H", "ids", "tlp") if st[k] is not None}
    return _plain_logprobs(st)


def _decode(codes, order, scale):
    """Pages [..., n_kv, 16 * hd] -> fp32 values [..., n_kv, 16, hd]."""
    u = codes.view(torch.uint8)[..., order]
    return u.view(torch.float8_e4m3fn).to(torch.float32).mul_(scale[..., None, None])


def _append(st):
    h, M = st["h"], st["M"]
    x = st["qkv"].float().view(M, h.nq + 2 * h.nkv, h.hd)
    half = h.hd // 2
    inv = torch.pow(torch.tensor(h.base, dtype=torch.float64, device="cuda"), torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / h.hd))
    ang = st["pos"].double()[:, None] * inv
    c, s = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    lo, hi = x[:, :h.nq + h.nkv, :half], x[:, :h.nq + h.nkv, half:]
    rot = torch.cat([lo * c - hi * s, hi * c + lo * s], -1)
    st["q"].copy_(rot[:, :h.nq])
    slot = st["pos"] % PAGE
    at = torch.arange(PAGE, device="cuda")[None, None, :, None]
    old, valid = at < st["held"][:, None, None, None], at < st["filled"][:, None, None, None]
    scales = st["scale"][st["ublk"]]
    new_scales = []
    for w, pool, order, new in ((0, st["k"], st["k_order"], rot[:, h.nq:]), (1, st["v"], st["v_order"], x[:, h.nq + h.nkv:])):
        codes = pool.view(torch.uint8)[st["ublk"]]
        val = torch.where(old, _decode(codes, order, scales[..., w]), 0.0)
        val[st["unit"], :, slot] = new
        most = val.abs().amax((2, 3)).double()
        mant, exp = torch.frexp(most / E4M3_MAX)          # most <= 448 * 2^k for the smallest k
        k = torch.where(mant > 0.5, exp, exp - 1).clamp(-100, 100)
        sc = torch.where(most > 0, torch.exp2(k.double()), 1.0).float()
        got = (val / sc[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        got = torch.where(valid, got, codes[..., order])
        codes[..., order.reshape(-1)] = got.reshape(got.shape[0], h.nkv, -1)
        pool.view(torch.uint8)[st["ublk"]] = codes
        new_scales.append(sc)
    st["scale"][st["ublk"]] = torch.stack(new_scales, -1)


def _attention(st):
    h, n, R = st["h"], st["n"], st["most_rows"]
    P = (st["most_tokens"] + PAGE - 1) // PAGE
    pages = st["pt"][:, :P].long().clamp(min=0)

    def held(pool, order, w):       # [n][n_kv][tokens][hd] in fp32
        u = pool.view(torch.uint8)[pages].transpose(1, 2).contiguous()[..., order]
        sc = st["scale"][pages][..., w].transpose(1, 2)
        return u.view(torch.float8_e4m3fn).to(torch.float32).mul_(sc[..., None, None]).view(n, h.nkv, P * PAGE, h.hd)

    rows = (st["off"][:n, None] + torch.arange(R, device="cuda")).clamp(max=st["M"] - 1)
    q = st["q"][rows].float().view(n, R, h.nkv, h.group, h.hd).transpose(1, 2).reshape(n, h.nkv, R * h.group, h.hd)
    s = torch.matmul(q, held(st["k"], st["k_order"], 0).transpose(2, 3)).mul_(1.0 / math.sqrt(h.hd)).view(n, h.nkv, R, h.group, P * PAGE)
    last = st["ctx"][:, None] + torch.arange(R, device="cuda")
    s.masked_fill_((torch.arange(P * PAGE, device="cuda") > last[..., None])[:, None, :, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    den = s.sum(-1)
    o = torch.matmul(s.view(n, h.nkv, R * h.group, P * PAGE), held(st["v"], st["v_order"], 1)).view(n, h.nkv, R, h.group, h.hd) / den[..., None]
    o = o.transpose(1, 2).reshape(n, R, h.nq, h.hd)
    return o[st["req"], st["row"]].to(h.torch)


def _plain_logprobs(st):
    on = st["tok"] >= 0
    x = st["x"].float() / st["T"]
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    s = e.sum(-1)
    lse = torch.log(s)
    lp = d.gather(1, st["tok"].clamp(min=0).long()[:, None])[:, 0] - lse
    H = lse - (e * d).sum(-1) / s
    st["lp"].copy_(torch.where(on, lp, st["lp"]))
    st["H"].copy_(torch.where(on, H, st["H"]))
    if st["top"]:
        at = torch.sort(st["x"], dim=-1, descending=True, stable=True)[1][:, :st["top"]]
        k = st["top"]
        st["ids"][:, :k] = torch.where(on[:, None], at.to(torch.int32), st["ids"][:, :k])
        st["tlp"][:, :k] = torch.where(on[:, None], d.gather(1, at) - lse[:, None], st["tlp"][:, :k])
    return {k: st[k] for k in ("lp", "H", "ids", "tlp") if st[k] is not None}


# ------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "logprobs":
        keep = np.random.default_rng([case["mix"], 31]).random(case["rows"]) < case["share"]
        keep[0] = True
        n, es = int(keep.sum()), 4 if case["dtype"] == "f32" else 2
        # a maximum, an exponential and three sums over each logit of the rows with a token
        return {"bytes": n * (case["vocab"] * es + 8 + 8 * case["top"]) + 4.0 * case["rows"], "flops": 6.0 * n * case["vocab"]}
    h = Heads(case["shape"])
    ctx, pre, gam = _lengths(case)
    nrow = (pre + gam + 1).astype(np.float64)
    M = nrow.sum()
    if case["kind"] == "append":
        held = (ctx % PAGE).astype(np.float64).sum()       # slots of the pages that are begun
        pages = ((ctx + nrow - 1) // PAGE - ctx // PAGE + 1).sum()
        kv = 2.0 * h.nkv * h.hd
        return {"bytes": M * ((h.nq + 2 * h.nkv) * h.hd * h.es + h.nq * h.hd * h.es + kv) + held * kv + pages * h.nkv * 16,
                "flops": M * (6.0 * (h.nq + h.nkv) * h.hd + 4.0 * kv)}
    tokens = ctx + nrow
    seen = (nrow * ctx + nrow * (nrow + 1) / 2).sum()       # (row, token) pairs
    kv = 2.0 * h.nkv * (h.hd + 4.0 / PAGE)
    return {"bytes": tokens.sum() * kv + 2.0 * M * h.nq * h.hd * h.es, "flops": seen * h.nq * (4.0 * h.hd + 5)}


# ------------------------------------------------------------------------------------------
# the operators in fp64, from their definition
# ------------------------------------------------------------------------------------------
def _exact_append(case, seed):
    st = _inputs(case, seed)
    h = st["h"]
    ctx, pre, gam = _lengths(case)
    off = st["off"].tolist()
    pools = [st["k"].to(torch.float64), st["v"].to(torch.float64)]
    scale = st["scale"].double()
    place = [st["k_order"], st["v_order"]]
    q = torch.empty(st["M"], h.nq, h.hd, dtype=torch.float64, device="cuda")
    freq = torch.tensor([h.base ** (-2.0 * i / h.hd) for i in range(h.hd // 2)], dtype=torch.float64, device="cuda")
    # e4m3's values in the order of their codes, the sign left out
    grid = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:-1],
                        dtype=torch.float64, device="cuda")

    def nearest(v):                 # ties to the even code
        a = v.abs()
        i = torch.searchsorted(grid, a.contiguous()).clamp(1, 126)
        below, above = a - grid[i - 1], grid[i] - a
        i = torch.where((below < above) | ((below == above) & (i % 2 == 1)), i - 1, i)
        return torch.where(v < 0, -grid[i], grid[i])

    for b in range(st["n"]):
        r0, r1 = off[b], off[b + 1]
        x = st["qkv"][r0:r1].double().view(r1 - r0, -1, h.hd)
        a = torch.arange(int(ctx[b]), int(ctx[b]) + r1 - r0, device="cuda").double()[:, None, None] * freq
        z = torch.complex(x[:, :h.nq + h.nkv, :h.hd // 2], x[:, :h.nq + h.nkv, h.hd // 2:]) * torch.polar(torch.ones_like(a), a)
        rot = torch.cat([z.real, z.imag], -1)
        q[r0:r1] = rot[:, :h.nq]
        p0, end = int(ctx[b]) // PAGE, int(ctx[b]) + r1 - r0
        blk = st["pt"][b, p0:(end + PAGE - 1) // PAGE].long()
        for w, new in ((0, rot[:, h.nq:]), (1, x[:, h.nq + h.nkv:])):
            held = int(ctx[b]) - p0 * PAGE
            page = pools[w][blk][..., place[w]]                      # [pages][n_kv][16][hd]
            tokens = (page * scale[blk][..., w, None, None]).transpose(1, 2).reshape(-1, h.nkv, h.hd).clone()
            tokens[held:end - p0 * PAGE] = new
            n = end - p0 * PAGE
            tokens[n:] = 0
            t = tokens.view(-1, PAGE, h.nkv, h.hd).transpose(1, 2)
            most = t.abs().amax((2, 3))
            k = torch.ceil(torch.log2(most / E4M3_MAX)).clamp(-100, 100)
            sc = torch.where(most > 0, torch.exp2(k), 1.0)
            got = nearest(t / sc[..., None, None])
            kept = (torch.arange(len(blk) * PAGE, device="cuda") < n).view(-1, 1, PAGE, 1)
            got = torch.where(kept, got, page)
            flat = pools[w][blk]
            flat[..., place[w].reshape(-1)] = got.reshape(len(blk), h.nkv, -1)
            pools[w][blk] = flat
            scale[blk, :, w] = sc
    return {"q": q, "k": pools[0], "v": pools[1], "scale": scale}


def _exact_attention(case, seed):
    st = _inputs(case, seed)
    h = st["h"]
    ctx, pre, gam = _lengths(case)
    off = st["off"].tolist()
    out = torch.empty(st["M"], h.nq, h.hd, dtype=torch.float64, device="cuda")
    for b in range(st["n"]):
        r0, r1 = off[b], off[b + 1]
        T = int(ctx[b]) + r1 - r0
        blk = st["pt"][b, :(T + PAGE - 1) // PAGE].long()
        for j in range(h.nkv):
            kv = []
            for w, pool, place in ((0, st["k"], st["k_order"]), (1, st["v"], st["v_order"])):
                page = pool.view(torch.uint8)[blk, j].view(torch.float8_e4m3fn).double() * st["scale"][blk, j, w].double()[:, None]
                kv.append(page[:, place].reshape(-1, h.hd)[:T])
            q = st["q"][r0:r1, j * h.group:(j + 1) * h.group].double()
            z = (q.reshape(-1, h.hd) @ kv[0].t().contiguous()).view(r1 - r0, h.group, T) / math.sqrt(h.hd)
            seen = torch.arange(T, device="cuda") <= (int(ctx[b]) + torch.arange(r1 - r0, device="cuda"))[:, None]
            p = torch.softmax(torch.where(seen[:, None], z, -math.inf), -1)
            out[r0:r1, j * h.group:(j + 1) * h.group] = (p.view(-1, T) @ kv[1]).view(r1 - r0, h.group, h.hd)
    return out


def _exact_logprobs(case, seed):
    st = _inputs(case, seed)
    res = {k: st[k].double() if st[k].is_floating_point() else st[k] for k in ("lp", "H", "ids", "tlp") if st[k] is not None}
    for a in range(0, st["x"].shape[0], 256):
        b = min(a + 256, st["x"].shape[0])
        on = (st["tok"][a:b] >= 0).nonzero()[:, 0]
        z = torch.log_softmax(st["x"][a:b][on].double() / st["T"], -1)
        res["lp"][a + on] = z.gather(1, st["tok"][a:b][on].long()[:, None])[:, 0]
        res["H"][a + on] = -(z.exp() * z).sum(-1)
        if st["top"]:
            top = torch.sort(z, dim=-1, descending=True)[0][:, :st["top"]]
            full = res["tlp"][a + on]
            full[:, :st["top"]] = top
            res["tlp"][a + on] = full
    if "ids" in res:
        res["ids"] = None            # which of equal logits comes first: no value in 64 bits
    return res


def _inputs(case, seed):
    """The state as the plain form has it."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    return {"append": _exact_append, "attention": _exact_attention, "logprobs": _exact_logprobs}[case["kind"]](case, seed)
