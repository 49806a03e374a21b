"""Measured cases of the operators around a KV cache that requests share and that outgrows its pool,
through the library's public entry points and in their plain form:

  wisp_attention_shared  one layer's ragged paged attention of a batch whose groups of requests share
                         a long prefix, and the log-sum-exp of every row's scores
  wisp_attention_mass    the attention weight that every cached token gets from the batch's rows,
                         accumulated with what it got before
  wisp_kv_evict          the tokens of least accumulated weight leave the cache: those kept move
                         together, their keys rotated to their new positions

The plain form is written in elementary torch operations in fp32 (angles, and sums over many rows, in
fp64), over batches padded to their longest request; `exact` states the same operators in fp64,
request by request.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

PAGE = 16
# query heads, kv heads, head_dim, storage, rotary base: the heads of the served model shapes
SHAPES = {
    "tiny": (4, 4, 64, "f32", 1e4),
    "8b": (32, 8, 128, "bf16", 5e5),
    "70b": (64, 8, 128, "bf16", 5e5),
}
STD = 1.15             # of rotated heads: what projections of unit-RMS rows give


class Heads:
    def __init__(self, key, layers=1):
        self.nq, self.nkv, self.hd, self.dtype, self.base = SHAPES[key]
        self.name, self.group = key, self.nq // self.nkv
        self.torch = torch.float32 if self.dtype == "f32" else torch.bfloat16
        self.es = 4 if self.dtype == "f32" else 2
        # what the library's model descriptor holds besides: not read by these operators
        self.n_layers, self.d_model, self.n_q_heads, self.n_kv_heads = layers, self.nq * self.hd, self.nq, self.nkv
        self.head_dim, self.d_ff, self.vocab, self.rms_eps, self.rope_base = self.hd, self.nq * self.hd, 1024, 1e-5, self.base


# ------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------
def _batch(name, kind, shape, groups, members, prefix, ctx, gamma, alone=0, new=0.0, prompt=(0, 0), plain=0.0, mix=1):
    """`groups` runs of requests that share a prefix of prefix tokens (in pages), `members` requests
    in each, then `alone` requests that share nothing; every request has ctx cached tokens of its
    own (log-uniform) and gamma drafts (a share `plain` of them none); a share `new` has none cached of
    its own and brings a prompt."""
    return dict(name=name, kind=kind, shape=shape, groups=groups, members_lo=members[0], members_hi=members[1],
                prefix_lo=prefix[0], prefix_hi=prefix[1], ctx_lo=ctx[0], ctx_hi=ctx[1], gamma_lo=gamma[0], gamma_hi=gamma[1],
                alone=alone, new=new, prompt_lo=prompt[0], prompt_hi=prompt[1], plain=plain, mix=mix)


def _evict(name, shape, layers, requests, ctx, keep, sink, recent, mix=1):
    """`requests` of ctx cached tokens (log-uniform), of which a share `keep` stays, the first `sink` and
    the last `recent` among them."""
    return dict(name=name, kind="evict", shape=shape, layers=layers, requests=requests, ctx_lo=ctx[0], ctx_hi=ctx[1],
                keep_lo=keep[0], keep_hi=keep[1], sink=sink, recent=recent, mix=mix)


def listed():
    return [
        # four chats on one system prompt, a layer's attention: the least that is worth sharing
        _batch("shared_8b_b4", "shared", "8b", 1, (4, 4), (1024, 1024), (64, 512), (5, 5)),
        # 32 chats on a longer one
        _batch("shared_8b_b32", "shared", "8b", 1, (32, 32), (2048, 2048), (128, 1024), (1, 8), mix=18),
        # 64 requests of a larger model about one document
        _batch("shared_70b_b64", "shared", "70b", 1, (64, 64), (8192, 8192), (64, 512), (1, 8), mix=3),
        # several system prompts, new questions among the running ones, and requests that share nothing
        _batch("shared_8b_groups", "shared", "8b", 3, (8, 16), (512, 4096), (16, 1024), (0, 8), alone=9, new=0.15, prompt=(20, 120),
               plain=0.25, mix=4),
        # 128 samples of one long prompt, plain decoding
        _batch("shared_8b_decode128", "shared", "8b", 1, (128, 128), (16384, 16384), (8, 256), (0, 0), mix=5),
        # a small fp32 model's sessions
        _batch("shared_tiny_f32", "shared", "tiny", 2, (8, 12), (256, 1024), (1, 300), (0, 8), alone=3, mix=6),
        # the weights of one session's tokens
        _batch("mass_8b_b1", "mass", "8b", 0, (0, 0), (0, 0), (4000, 4000), (5, 5), alone=1),
        # of 32 sessions about one document
        _batch("mass_8b_shared32", "mass", "8b", 1, (32, 32), (4096, 4096), (256, 2048), (1, 8), mix=8),
        # of a long prompt, as it enters the cache, with a few sessions in its batch
        _batch("mass_8b_prefill", "mass", "8b", 0, (0, 0), (0, 0), (300, 2000), (1, 5), alone=4, new=0.25, prompt=(4096, 4096), mix=9),
        # one session's cache back to a quarter, a layer
        _evict("evict_8b_b1", "8b", 1, 1, (8000, 8000), (0.25, 0.25), 64, 256),
        # 32 sessions' to about half, two layers
        _evict("evict_8b_b32", "8b", 2, 32, (2048, 8192), (0.4, 0.6), 64, 256, mix=11),
        # a small fp32 model's, odd lengths
        _evict("evict_tiny_f32", "tiny", 2, 12, (100, 3000), (0.2, 0.9), 5, 13, mix=13),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"shared": 90e9, "mass": 45e9, "evict": 1.2e9}
    while True:
        kind = rng.choices(["shared", "mass", "evict"], [4, 3, 3])[0]
        shape = rng.choices(["8b", "70b", "tiny"], [5, 2, 2])[0]
        mix = rng.randrange(1, 1 << 30)
        if kind == "evict":
            hi = _log_int(rng, 40, 16384)
            keep = rng.uniform(0.1, 0.9)
            c = _evict("", "8b" if shape == "70b" else shape, rng.randint(1, 4), _log_int(rng, 1, 64), (max(20, int(hi * rng.uniform(0.1, 1.0))), max(20, hi)),
                       (keep, min(1.0, keep + rng.uniform(0.0, 0.2))), rng.choice([0, 1, 4, 16, 64, rng.randint(0, 100)]), rng.randint(0, 300), mix=mix)
        else:
            groups = rng.choice([0, 1, 1, 1, 2, 3, 5])
            hi, pre = _log_int(rng, 4, 4096), PAGE * _log_int(rng, 1, 1024)
            m_hi = _log_int(rng, 2, 96)
            g_hi = rng.randint(0, 12)
            p_hi = _log_int(rng, 10, 300 if groups else 2000)
            c = _batch("", kind, shape, groups, (max(1, int(m_hi * rng.uniform(0.2, 1.0))), m_hi) if groups else (0, 0),
                       (max(PAGE, int(pre * rng.uniform(0.1, 1.0))), pre) if groups else (0, 0), (max(1, int(hi * rng.uniform(0.05, 1.0))), hi),
                       (rng.randint(0, g_hi), g_hi), alone=_log_int(rng, 1, 24) if not groups else rng.choice([0, 0, 1, 4, 10]),
                       new=rng.choice([0.0, 0.0, 0.1, 0.3]), prompt=(max(1, int(p_hi * rng.uniform(0.1, 1.0))), p_hi),
                       plain=rng.choice([0.0, 0.25]), mix=mix)
        c.pop("name")
        w = work(c)
        # the plain form is padded to the longest request: what it pads may not grow without bound
        if kind != "evict":
            ctx, pre_, gam, _, _ = _lengths(c)
            rows, h = pre_ + gam + 1, Heads(c["shape"])
            padded = len(ctx) * int((ctx + rows).max())
            if padded > 2_200_000 or padded * int(rows.max()) * h.nq > 700_000_000:
                continue
        if (w["bytes"] if kind == "evict" else w["flops"]) <= most[kind]:
            return c


def _log_ints(r, lo, hi, n):
    return np.clip(np.rint(np.exp(r.uniform(math.log(max(lo, 1)), math.log(max(hi, 1)), n))), lo, hi).astype(np.int32)


def _lengths(case):
    """(cached tokens, prompt rows, drafts) of each request, then each group's requests and shared
    tokens, from the case alone."""
    r = np.random.default_rng([case["mix"], 907])
    size = r.integers(case["members_lo"], case["members_hi"], case["groups"], endpoint=True).astype(np.int32)
    prefix = _log_ints(r, case["prefix_lo"], case["prefix_hi"], case["groups"]) // PAGE * PAGE
    size = np.concatenate([size, np.ones(case["alone"], np.int32)]).astype(np.int32)
    prefix = np.concatenate([prefix, np.zeros(case["alone"], np.int32)]).astype(np.int32)
    n = int(size.sum())
    ctx, pre = _log_ints(r, case["ctx_lo"], case["ctx_hi"], n), np.zeros(n, np.int32)
    gam = r.integers(case["gamma_lo"], case["gamma_hi"], n, endpoint=True).astype(np.int32)
    gam = np.where(r.random(n) < case["plain"], 0, gam).astype(np.int32)
    new = r.random(n) < case["new"]
    pre[new] = _log_ints(r, case["prompt_lo"], case["prompt_hi"], n)[new]
    ctx[new] = 0
    return (ctx + np.repeat(prefix, size)).astype(np.int32), pre, gam, size, prefix


def _counted(case):
    """The rows of each request whose weights count: the prompt, the root and the accepted drafts."""
    _, pre, gam, _, _ = _lengths(case)
    return pre + 1 + np.minimum(np.random.default_rng([case["mix"], 919]).integers(0, 9, len(gam)), gam).astype(np.int32)


def _kept(case):
    """(cached tokens, kept tokens) of each request, from the case alone."""
    r = np.random.default_rng([case["mix"], 911])
    ctx = _log_ints(r, case["ctx_lo"], case["ctx_hi"], case["requests"])
    keep = np.rint(ctx * r.uniform(case["keep_lo"], case["keep_hi"], case["requests"])).astype(np.int32)
    return ctx, np.minimum(np.maximum(keep, case["sink"] + case["recent"]), ctx).astype(np.int32)


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) & ((1 << 62) - 1))
    return g


def _normal(shape, std, dtype, g):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)


def _page_tables(seed, *tokens):
    """Scattered pages for each of the lists of token counts: parts of one permutation of a pool; -1 past
    a request's last page."""
    needs = [(np.asarray(t, np.int64) + PAGE - 1) // PAGE for t in tokens]
    n_blocks = int(sum(k.sum() for k in needs)) + 3
    perm = np.random.default_rng([int(seed), 7]).permutation(n_blocks).astype(np.int32)
    tabs, o = [], 0
    for need in needs:
        tab = np.full((len(need), max(int(need.max(initial=0)), 1)), -1, np.int32)
        for i, k in enumerate(need):
            tab[i, :k] = perm[o:o + k]
            o += k
        tabs.append(tab)
    return tabs, n_blocks


def _k_order(hd):
    """[16][hd] -> place of (slot, dim) in a K page."""
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return (((e // 32) * 2 + (s // 4) % 2) * 4 + (e % 32) // 8) * 64 + ((s // 8) * 4 + s % 4) * 8 + e % 8


def _v_order(hd):
    """[16][hd] -> place of (slot, dim) in a V page."""
    s, e = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return ((e // 16) * 2 + s // 8) * 128 + (e % 16) * 8 + s % 8


def _ints(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int64), device="cuda")


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32), device="cuda")


def prepare(case, seed):
    return _prepare_evict(case, seed) if case["kind"] == "evict" else _prepare_batch(case, seed)


def _prepare_batch(case, seed):
    h = Heads(case["shape"])
    ctx, pre, gam, size, prefix = _lengths(case)
    nrow = pre + gam + 1
    of = np.repeat(np.arange(len(size)), size)              # a request's group
    (common, tail), n_blocks = _page_tables(seed, prefix, ctx + nrow - prefix[of])
    tab = np.full((len(ctx), int((ctx + nrow + PAGE - 1).max() // PAGE)), -1, np.int32)
    for i, g in enumerate(of):
        k, t = prefix[g] // PAGE, tail[i][tail[i] >= 0]
        tab[i, :k], tab[i, k:k + len(t)] = common[g, :k], t
    off = np.concatenate([[0], np.cumsum(nrow)])
    M = int(off[-1])
    req = np.repeat(np.arange(len(ctx)), nrow)
    g = _gen(seed, 2)
    pages = (n_blocks, h.nkv, PAGE * h.hd)
    st = dict(kind=case["kind"], h=h, k=_normal(pages, STD, h.torch, g), v=_normal(pages, STD, h.torch, g), M=M, n=len(ctx),
              pt=_i32(tab), ctx=_ints(ctx), off=_ints(off), nrow=_ints(nrow), req=_ints(req), row=_ints(np.arange(M) - off[req]),
              most_rows=int(nrow.max()), most_tokens=int((ctx + nrow).max()), k_order=_ints(_k_order(h.hd)), v_order=_ints(_v_order(h.hd)))
    st["q"] = _normal((M, h.nq, h.hd), STD, h.torch, _gen(seed, 3))
    st["lse"] = torch.empty(M, h.nq, device="cuda")
    if case["kind"] == "shared":
        st["out"] = torch.empty_like(st["q"])
    else:
        st["lse"].copy_(_row_lse(st))
        # what the tokens got before, of some steps
        st["prev"] = torch.empty(n_blocks, h.nkv, PAGE, device="cuda").exponential_(50.0, generator=_gen(seed, 4))
        st["mass"] = torch.zeros(n_blocks, h.nkv, PAGE, device="cuda")
        st["count"] = _i32(_counted(case))
        st["decay"] = 0.98
    if own:
        import paper_2601_11652_amd as W
        model = W.GpuModel.shape_only(h)
        desc = W.BatchDesc(ctx, gam, st["pt"], 1.0, None, pre if pre.any() else None)
        st["kv"] = W.KVPool(st["k"][None], st["v"][None])
        ws = W.workspace(W.wisp_shared_workspace_size(model, desc, size, prefix))
        st["plan"] = W.wisp_shared_plan(model, desc, size, prefix, ws)
    return st


def _prepare_evict(case, seed):
    h = Heads(case["shape"], case["layers"])
    ctx, keep = _kept(case)
    (tab, to), n_blocks = _page_tables(seed, ctx, keep)
    # the pages of tokens that do not move stay where they are
    fixed = min(case["sink"] // PAGE, to.shape[1], tab.shape[1])
    for i in range(len(ctx)):
        k = min(fixed, int(keep[i]) // PAGE)
        to[i, :k] = tab[i, :k]
    g = _gen(seed, 2)
    pages = (h.n_layers, n_blocks, h.nkv, PAGE * h.hd)
    st = dict(kind="evict", h=h, n=len(ctx), k=_normal(pages, STD, h.torch, g), v=_normal(pages, STD, h.torch, g),
              # a token's weight: a few have most of it
              mass=torch.empty(pages[:3] + (PAGE,), device="cuda").log_normal_(-2.0, 2.0, generator=g),
              pt=_i32(tab), to=_i32(to), ctx=_ints(ctx), keep=_ints(keep), most=int(ctx.max()), most_kept=int(keep.max()),
              sink=case["sink"], recent=case["recent"], k_order=_ints(_k_order(h.hd)), v_order=_ints(_v_order(h.hd)),
              start=_ints(np.concatenate([[0], np.cumsum(keep)])), total=int(keep.sum()),
              kept=torch.full((h.n_layers, h.nkv, int(keep.sum())), -1, dtype=torch.int32, device="cuda"))
    if own:
        import paper_2601_11652_amd as W
        st["model"], st["kv"] = W.GpuModel.shape_only(h), W.KVPool(st["k"], st["v"])
        st["desc"] = W.BatchDesc(ctx, np.zeros(len(ctx), np.int32), st["pt"])
        st["counts"] = (keep, np.full(len(ctx), case["sink"], np.int32), np.full(len(ctx), case["recent"], np.int32))
        st["ws"] = W.workspace(W.wisp_kv_evict_workspace_size(st["model"], st["desc"]))
    return st


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(st):
    if own:
        import paper_2601_11652_amd as W
    if st["kind"] == "shared":
        if not own:
            return dict(zip(("out", "lse"), _attention(st)))
        W.wisp_attention_shared(st["plan"], st["kv"], st["q"], st["out"], st["lse"])
        return {"out": st["out"], "lse": st["lse"]}
    if st["kind"] == "mass":
        if not own:
            return _mass(st)
        W.wisp_attention_mass(st["plan"], st["kv"], st["q"], st["lse"], st["mass"], st["prev"], st["decay"], st["count"])
        return st["mass"]
    if own:
        keep, sink, recent = st["counts"]
        W.wisp_kv_evict(st["model"], st["kv"], st["desc"], keep, st["mass"], st["kept"], st["ws"], sink, recent, st["to"])
    else:
        _move(st)
    return {name: st[name] for name in ("k", "v", "mass", "kept")}


def _held(st, pool, order):
    """Every request's tokens [n][n_kv][tokens][hd] in fp32, padded to the longest."""
    h, P = st["h"], (st["most_tokens"] + PAGE - 1) // PAGE
    x = pool[st["pt"][:, :P].long().clamp(min=0)].transpose(1, 2).contiguous()
    return x[..., order].float().view(st["n"], h.nkv, P * PAGE, h.hd)


def _scores(st):
    """[n][n_kv][rows][group][tokens], -inf where a row does not see a token."""
    h, n, R = st["h"], st["n"], st["most_rows"]
    rows = (st["off"][:n, None] + torch.arange(R, device="cuda")).clamp(max=st["M"] - 1)
    q = st["q"][rows].float().view(n, R, h.nkv, h.group, h.hd).transpose(1, 2).reshape(n, h.nkv, R * h.group, h.hd)
    k = _held(st, st["k"], st["k_order"])
    s = torch.matmul(q, k.transpose(2, 3)).mul_(1.0 / math.sqrt(h.hd)).view(n, h.nkv, R, h.group, -1)
    last = st["ctx"][:, None] + torch.arange(R, device="cuda")
    return s.masked_fill_((torch.arange(k.shape[2], device="cuda") > last[..., None])[:, None, :, None], -math.inf)


def _by_row(st, x):
    """[n][n_kv][rows][group][...] -> [M][n_q][...]"""
    x = x.transpose(1, 2)[st["req"], st["row"]]
    return x.reshape(st["M"], st["h"].nq, *x.shape[3:])


def _attention(st):
    h = st["h"]
    s = _scores(st)
    m = s.amax(-1, keepdim=True)
    e = s.sub_(m).exp_()
    den = e.sum(-1)
    n, _, R, _, T = e.shape
    o = torch.matmul(e.view(n, h.nkv, R * h.group, T), _held(st, st["v"], st["v_order"])).view(n, h.nkv, R, h.group, h.hd)
    return _by_row(st, o / den[..., None]).to(h.torch), _by_row(st, m[..., 0] + torch.log(den))


def _row_lse(st):
    s = _scores(st)
    m = s.amax(-1, keepdim=True)
    return _by_row(st, m[..., 0] + torch.log(s.sub_(m).exp_().sum(-1)))


def _mass(st):
    h, n, R = st["h"], st["n"], st["most_rows"]
    s = _scores(st)
    rows = (st["off"][:n, None] + torch.arange(R, device="cuda")).clamp(max=st["M"] - 1)
    lse = st["lse"][rows].view(n, R, h.nkv, h.group).transpose(1, 2)
    p = s.sub_(lse[..., None]).exp_()
    p.masked_fill_((torch.arange(R, device="cuda") >= st["count"][:, None])[:, None, :, None, None], 0.0)
    got = p.sum((2, 3), dtype=torch.float64).transpose(1, 2)                    # [n][tokens][n_kv]
    t = torch.arange(got.shape[1], device="cuda")
    page = st["pt"][:, :got.shape[1] // PAGE].long().repeat_interleave(PAGE, 1)
    place = page * PAGE + t % PAGE
    new = t < (st["ctx"] + st["nrow"])[:, None]
    total = torch.zeros(st["mass"].shape[0] * PAGE, h.nkv, dtype=torch.float64, device="cuda")
    total.index_add_(0, place[new], got[new])
    decay = torch.zeros(total.shape[0], 1, dtype=torch.float64, device="cuda")
    decay[place[t < st["ctx"][:, None]]] = st["decay"]
    prev = st["prev"].transpose(1, 2).reshape(-1, h.nkv)
    val = (prev * decay + total).float().view(-1, PAGE, h.nkv).transpose(1, 2)
    on = torch.zeros(total.shape[0], dtype=torch.bool, device="cuda")
    on[place[new]] = True
    st["mass"].copy_(torch.where(on.view(-1, 1, PAGE), val, st["mass"]))
    return st["mass"]


def _move(st):
    h, L, n, T, K = st["h"], st["h"].n_layers, st["n"], st["most"], st["most_kept"]
    pos = torch.arange(T, device="cuda")
    held = st["pt"][:, pos // PAGE].long().clamp(min=0)                         # [n][T]
    mass = st["mass"][:, held, :, (pos % PAGE)[None]]                          # [n][T][L][n_kv]: advanced dims first
    mass = mass.permute(2, 3, 0, 1)
    ctx = st["ctx"][:, None]
    fixed = (pos < st["sink"]) | (pos >= ctx - st["recent"])
    key = torch.where(fixed & (pos < ctx), math.inf, mass).masked_fill(pos >= ctx, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    rank = torch.empty_like(order).scatter_(-1, order, pos.expand_as(order).contiguous())
    chosen = rank < st["keep"][:, None]
    src = torch.sort(torch.where(chosen, pos, T), dim=-1)[0][..., :K]          # [L][n_kv][n][K], T past a request's last
    to = torch.arange(K, device="cuda")
    valid = to < st["keep"][:, None]                                           # [n][K]
    at = src.clamp(max=T - 1)
    layer, head = torch.arange(L, device="cuda")[:, None, None, None], torch.arange(h.nkv, device="cuda")[:, None, None]
    page = st["pt"][torch.arange(n, device="cuda")[:, None], at // PAGE].long()
    k = st["k"][..., st["k_order"]][layer, page, head, at % PAGE].float()      # [L][n_kv][n][K][hd]
    v = st["v"][..., st["v_order"]][layer, page, head, at % PAGE]
    got = st["mass"][layer, page, head, at % PAGE]
    half = h.hd // 2
    inv = torch.pow(torch.tensor(h.base, dtype=torch.float64, device="cuda"), torch.arange(half, device="cuda", dtype=torch.float64) * (-2.0 / h.hd))
    ang = (to - at).double()[..., None] * inv
    c, s = torch.cos(ang).float(), torch.sin(ang).float()
    k = torch.cat([k[..., :half] * c - k[..., half:] * s, k[..., half:] * c + k[..., :half] * s], -1).to(h.torch)
    where = st["to"][:, to // PAGE].long()
    r, i = valid.nonzero(as_tuple=True)
    b, slot = where[r, i], to[i] % PAGE
    for name, x, order in (("k", k, st["k_order"]), ("v", v, st["v_order"])):
        st[name][layer, b[:, None], head, order[slot]] = x[:, :, r, i]
    st["mass"][:, b, :, slot] = got[:, :, r, i].permute(2, 0, 1)
    st["kept"].copy_(src[:, :, r, i])


# ------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "evict":
        h = Heads(case["shape"], case["layers"])
        ctx, keep = (x.astype(np.float64) for x in _kept(case))
        # kept tokens move, but for those of the first pages, which keep their places
        moved = (keep - np.minimum(case["sink"] // PAGE, keep // PAGE) * PAGE).sum() * h.n_layers * h.nkv
        return {"bytes": moved * (4.0 * h.hd * h.es + 4) + (4.0 * ctx.sum() + 4.0 * keep.sum()) * h.n_layers * h.nkv, "flops": moved * 3.0 * h.hd}
    h = Heads(case["shape"])
    ctx, pre, gam, size, prefix = _lengths(case)
    nrow = (pre + gam + 1).astype(np.float64)
    tokens = float(prefix.sum() + (ctx + nrow).sum() - (prefix * size).sum())   # a group's shared ones once
    if case["kind"] == "shared":
        seen = (nrow * ctx + nrow * (nrow + 1) / 2).sum()      # (row, token) pairs
        return {"bytes": tokens * 2.0 * h.nkv * h.hd * h.es + nrow.sum() * h.nq * (2.0 * h.hd * h.es + 4), "flops": seen * h.nq * (4.0 * h.hd + 5)}
    c = _counted(case).astype(np.float64)
    seen = (c * ctx + c * (c + 1) / 2).sum()
    return {"bytes": tokens * h.nkv * (h.hd * h.es + 8.0) + c.sum() * h.nq * (h.hd * h.es + 4.0), "flops": seen * h.nq * (2.0 * h.hd + 3)}


# ------------------------------------------------------------------------------------------
# the operators in fp64, from their definition
# ------------------------------------------------------------------------------------------
def _tokens(st, pool, order, b, j, T):
    """The first T tokens of request b, kv head j, [T][hd] in fp64."""
    blk = st["pt"][b, :(T + PAGE - 1) // PAGE].long()
    return pool[blk, j].double()[:, order].reshape(-1, st["h"].hd)[:T]


def _exact_batch(case, seed):
    st = _inputs(case, seed)
    h, off, ctx = st["h"], st["off"].tolist(), st["ctx"].tolist()
    mass = case["kind"] == "mass"
    out = torch.empty(0 if mass else st["M"], h.nq, h.hd, dtype=torch.float64, device="cuda")
    lse = torch.empty(0 if mass else st["M"], h.nq, dtype=torch.float64, device="cuda")
    pool = st["mass"].double() if mass else None
    count = _counted(case) if mass else None
    # a page's slots before this batch: what they got before, less the decay; new slots start at nothing
    if mass:
        for b in range(st["n"]):
            for a, e, f in ((0, ctx[b], st["decay"]), (ctx[b], ctx[b] + off[b + 1] - off[b], 0.0)):
                t = torch.arange(a, e, device="cuda")
                blk = st["pt"][b, t // PAGE].long()
                pool[blk, :, t % PAGE] = f * st["prev"][blk, :, t % PAGE].double()
    for b in range(st["n"]):
        r0, r1 = off[b], off[b + 1]
        T = ctx[b] + r1 - r0
        t = torch.arange(T, device="cuda")
        seen = t <= (ctx[b] + torch.arange(r1 - r0, device="cuda"))[:, None]
        for j in range(h.nkv):
            q = st["q"][r0:r1, j * h.group:(j + 1) * h.group].double()
            z = (q.reshape(-1, h.hd) @ _tokens(st, st["k"], st["k_order"], b, j, T).t().contiguous()).view(r1 - r0, h.group, T) / math.sqrt(h.hd)
            z = torch.where(seen[:, None], z, -math.inf)
            if mass:
                n = int(count[b])
                p = torch.exp(z[:n] - st["lse"][r0:r0 + n, j * h.group:(j + 1) * h.group, None].double())
                pool[st["pt"][b, t // PAGE].long(), j, t % PAGE] += p.sum((0, 1))
            else:
                lse[r0:r1, j * h.group:(j + 1) * h.group] = torch.logsumexp(z, -1)
                v = _tokens(st, st["v"], st["v_order"], b, j, T)
                out[r0:r1, j * h.group:(j + 1) * h.group] = (torch.softmax(z, -1).view(-1, T) @ v).view(r1 - r0, h.group, h.hd)
    return pool if mass else {"out": out, "lse": lse}


def _exact_evict(case, seed):
    st = _inputs(case, seed)
    h = st["h"]
    ctx, keep = _kept(case)
    res = {"k": st["k"].double(), "v": st["v"].double(), "mass": st["mass"].double(), "kept": st["kept"].clone()}
    mass = st["mass"].cpu().numpy()
    pt, start = st["pt"].cpu().numpy(), np.concatenate([[0], np.cumsum(keep)])
    freq = torch.tensor([h.base ** (-2.0 * i / h.hd) for i in range(h.hd // 2)], dtype=torch.float64, device="cuda")
    for b in range(st["n"]):
        T, n = int(ctx[b]), int(keep[b])
        blk, to = st["pt"][b, :(T + PAGE - 1) // PAGE].long(), st["to"][b, :(n + PAGE - 1) // PAGE].long()
        for layer in range(h.n_layers):
            for j in range(h.nkv):
                if n < T:
                    w = mass[layer, pt[b, :len(blk)], j].reshape(-1)[:T]
                    middle = np.arange(st["sink"], T - st["recent"])
                    best = middle[np.argsort(-w[middle], kind="stable")[:n - st["sink"] - st["recent"]]]
                    src = np.sort(np.concatenate([np.arange(st["sink"]), best, np.arange(T - st["recent"], T)]))
                else:
                    src = np.arange(T)
                at = _ints(src)
                a = (torch.arange(n, device="cuda") - at).double()[:, None] * freq
                k = st["k"][layer, blk, j].double()[:, st["k_order"]].reshape(-1, h.hd)[at]
                z = torch.complex(k[:, :h.hd // 2], k[:, h.hd // 2:]) * torch.polar(torch.ones_like(a), a)
                v = st["v"][layer, blk, j].double()[:, st["v_order"]].reshape(-1, h.hd)[at]
                page, slot = to[torch.arange(n, device="cuda") // PAGE, None], torch.arange(n, device="cuda") % PAGE
                res["k"][layer, page, j, st["k_order"][slot]] = torch.cat([z.real, z.imag], -1)
                res["v"][layer, page, j, st["v_order"][slot]] = v
                res["mass"][layer, page[:, 0], j, slot] = st["mass"][layer, blk, j].reshape(-1)[at].double()
                res["kept"][layer, j, start[b]:start[b + 1]] = at.to(torch.int32)
    return res


def exact(case, seed):
    return _exact_evict(case, seed) if case["kind"] == "evict" else _exact_batch(case, seed)


def _inputs(case, seed):
    """The state as the plain form has it."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was
