"""Eviction from the cache by accumulated weight, against fp64."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from gpu_harness import log, to_dev
from oracle import shared
from shared_harness import HALF, U, bits, from_pages, shape, to_pages, torch_type

pytestmark = pytest.mark.gpu


class Cache:
    """Requests of ctx tokens in scattered pages of a pool of `layers`; pages of none hold NaN."""

    def __init__(self, ctx, n_kv, hd, bf16, seed, layers=1, base=1e4, spare=0):
        self.rng = rng = np.random.default_rng(seed)
        self.ctx, self.n_kv, self.hd, self.bf16, self.layers, self.base = np.asarray(ctx, np.int32), n_kv, hd, bf16, layers, base
        self.model = W.GpuModel.shape_only(shape(n_kv, n_kv, hd, bf16, layers, base))
        need = (self.ctx + 15) // 16
        self.nb = int(need.sum()) + 2 + spare
        self.perm = rng.permutation(self.nb).astype(np.int32)
        self.pt = np.full((len(self.ctx), max(int(need.max()), 1) + 1), -1, np.int32)
        o = 0
        for i, k in enumerate(need):
            self.pt[i, :k] = self.perm[o:o + k]
            o += int(k)
        self.free = self.perm[o:]
        shp = (layers, self.nb, n_kv, 16, hd)
        round_ = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch_type(bf16)).double().numpy()
        self.k, self.v = round_(rng.normal(0, 1.2, shp)), round_(rng.normal(0, 1.2, shp))
        self.mass = rng.lognormal(-2, 2, shp[:4]).astype(np.float32)
        self.k[:, self.free], self.v[:, self.free], self.mass[:, self.free] = np.nan, np.nan, np.nan
        self.desc = W.BatchDesc(self.ctx, np.zeros(len(self.ctx), np.int32), to_dev(self.pt))

    def to_dev(self):
        self.kv = W.KVPool(to_pages(self.k, "k", self.bf16), to_pages(self.v, "v", self.bf16))
        self.dm = to_dev(self.mass)
        return self

    def run(self, keep, sink=None, recent=None, to=None, stream=None):
        keep = np.asarray(keep, np.int32)
        total = int(np.minimum(keep, self.ctx).sum())
        kept = torch.full((self.layers, self.n_kv, total), -9, dtype=torch.int32, device="cuda")
        ws = W.workspace(W.wisp_kv_evict_workspace_size(self.model, self.desc))
        W.wisp_kv_evict(self.model, self.kv, self.desc, keep, self.dm, kept, ws, sink, recent, None if to is None else to_dev(to), stream)
        W.wisp_check(ws)
        return kept.cpu().numpy()

    def check(self, kept, keep, sink=None, recent=None, to=None):
        """Against the oracle from the state that the host arrays hold; they then hold the new one."""
        zero = np.zeros(len(self.ctx), np.int32)
        sink, recent, to = zero if sink is None else sink, zero if recent is None else recent, self.pt if to is None else to
        k0, v0, m0 = self.k.copy(), self.v.copy(), self.mass.copy()
        want, pair = shared.evict(self.k, self.v, self.mass, self.pt, self.ctx, keep, sink, recent, to, self.base)
        np.testing.assert_array_equal(kept, want)
        gk, gv = from_pages(self.kv.k, "k", self.hd), from_pages(self.kv.v, "v", self.hd)
        exact = lambda a: bits(torch.from_numpy(np.ascontiguousarray(a)).to(torch_type(self.bf16)))
        np.testing.assert_array_equal(bits(gv), exact(self.v))
        np.testing.assert_array_equal(self.dm.cpu().numpy().view(np.int32), self.mass.view(np.int32))
        still = pair == 0
        np.testing.assert_array_equal(bits(gk)[still], exact(self.k)[still])
        # an angle is off by half a step of half a turn in fp32, 3.2 half steps; sine and cosine by 2 more; two
        # products and their sum by 3, and the result is rounded once
        h = HALF[self.bf16]
        bound = h * np.abs(self.k) + 10 * U * (1 + h) * pair
        off = np.abs(gk.double().numpy() - self.k)
        assert np.all(off[~still] <= bound[~still]), (off[~still] / bound[~still]).max()
        self.k = gk.double().numpy()
        return k0, v0, m0


CASES = [
    # ctx, kv heads, head_dim, bf16, layers; keep; sink; recent
    ([40], 1, 64, True, 1, [17], [0], [0]),
    ([1], 2, 64, True, 1, [0], None, None),
    ([1, 2, 3], 2, 64, False, 1, [1, 1, 3], None, None),
    ([100, 33, 0, 16, 17], 2, 128, True, 2, [50, 20, 5, 3, 16], [4, 0, 0, 1, 16], [10, 20, 0, 2, 0]),
    ([300, 257], 8, 128, True, 1, [64, 256], [20, 16], [7, 0]),
    ([5000, 40, 1030], 2, 64, True, 2, [1234, 40, 1029], [16, 3, 0], [100, 0, 1]),
    ([2100], 1, 128, True, 1, [700], [33], [64]),
    ([200, 90], 3, 32, False, 3, [100, 13], [5, 3], [13, 10]),
    ([129], 2, 96, False, 1, [77], [1], [1]),
    ([150], 1, 160, False, 2, [31], [16], [15]),
    ([70], 2, 192, False, 1, [69], None, [68]),
    ([64], 1, 224, False, 1, [32], [32], None),
    ([333], 2, 256, False, 1, [160], [10], [10]),
    ([20000], 1, 64, True, 1, [9000], [64], [256]),           # more than the selection holds in LDS
]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_evict_matches_oracle(case, in_place):
    ctx, n_kv, hd, bf16, layers, keep, sink, recent = CASES[case]
    log(f"evict {CASES[case]} in place {in_place}")
    kept_tokens = np.minimum(keep, ctx)
    c = Cache(ctx, n_kv, hd, bf16, 500 + case, layers, spare=0 if in_place else int(((kept_tokens + 15) // 16).sum())).to_dev()
    to = None
    if not in_place:
        to = np.full((len(ctx), max(int((kept_tokens.max() + 15) // 16), 1)), -1, np.int32)
        o = 0
        for i, n in enumerate((kept_tokens + 15) // 16):
            to[i, :n] = c.free[o:o + n]
            o += int(n)
        if sink is not None:                                  # pages of the first tokens stay where they are
            for i, s in enumerate(sink):
                to[i, :s // 16] = c.pt[i, :s // 16]
    kept = c.run(keep, sink, recent, to)
    c.check(kept, keep, sink, recent, to)


def test_again_and_again_in_place():
    """Evicted, evicted again, with the lengths that the first one left."""
    c = Cache([400, 90, 17], 2, 64, True, 7, layers=2).to_dev()
    for keep in ([300, 80, 17], [111, 33, 16], [20, 33, 1]):
        kept = c.run(keep, [2, 16, 0], [5, 3, 1])
        c.check(kept, keep, [2, 16, 0], [5, 3, 1])
        c.ctx = np.minimum(keep, c.ctx).astype(np.int32)
        c.desc = W.BatchDesc(c.ctx, np.zeros(3, np.int32), to_dev(c.pt))


def test_ties_infinities_and_nan():
    """Equal weights: the first ones stay; -0 is 0; NaN goes before -infinity; weights of both signs."""
    c = Cache([200, 200, 200, 200], 1, 64, False, 8)
    values = [np.zeros(200, np.float32), np.tile(np.array([0.0, -0.0, 1.0, 1.0], np.float32), 50),
              np.where(np.arange(200) % 3 == 0, np.nan, np.where(np.arange(200) % 3 == 1, -np.inf, np.inf)).astype(np.float32),
              c.rng.normal(0, 1, 200).astype(np.float32)]
    for b, w in enumerate(values):
        for t in range(200):
            c.mass[0, c.pt[b, t // 16], 0, t % 16] = w[t]
    c.to_dev()
    keep = [70, 120, 150, 33]
    kept = c.run(keep, [0, 3, 1, 0], [0, 5, 1, 0])
    c.check(kept, keep, [0, 3, 1, 0], [0, 5, 1, 0])
    np.testing.assert_array_equal(kept[0, 0, :70], np.arange(70))


def test_values_that_are_not_finite_move_as_they_are():
    c = Cache([64], 1, 64, True, 9)
    c.v[0, c.pt[0, 2], 0, 5, 7] = np.nan
    c.v[0, c.pt[0, 3], 0, 1, 9] = -np.inf
    c.k[0, c.pt[0, 0], 0, 1, 3] = np.inf                      # a token that stays where it is
    c.to_dev()
    kept = c.run([60], [2], [40])
    c.check(kept, [60], [2], [40])


def test_all_stay():
    """keep of ctx_len or more: nothing in place changes, a copy is exact."""
    c = Cache([37, 16], 2, 64, True, 10, spare=5).to_dev()
    before = [bits(t.cpu()) for t in (c.kv.k, c.kv.v)]
    kept = c.run([37, 99], [50, 0], [50, 0])
    np.testing.assert_array_equal(kept[0, 0], np.r_[0:37, 0:16])
    for a, t in zip(before, (c.kv.k, c.kv.v)):
        np.testing.assert_array_equal(a, bits(t.cpu()))
    to = np.full((2, 3), -1, np.int32)
    to[0], to[1, 0] = c.free[:3], c.free[3]
    kept = c.run([37, 99], None, None, to)
    c.check(kept, [37, 99], None, None, to)


def test_bad_pages_are_reported_and_not_written():
    c = Cache([100, 60], 2, 64, True, 11).to_dev()
    for bad in (-1, c.nb, 2 ** 31 - 1):
        tab = c.pt.copy()
        tab[0, 1] = bad
        c.desc.page_table.copy_(to_dev(tab))
        kept = torch.zeros(1, 2, 60, dtype=torch.int32, device="cuda")
        ws = W.workspace(W.wisp_kv_evict_workspace_size(c.model, c.desc))
        W.wisp_kv_evict(c.model, c.kv, c.desc, [40, 20], c.dm, kept, ws)
        with pytest.raises(W.WispError) as e:
            W.wisp_check(ws)
        assert e.value.status == W.WISP_E_DEVICE_INPUT
    free = torch.from_numpy(c.free.astype(np.int64)).cuda()
    assert torch.isnan(c.kv.k[0, free].float()).all() and torch.isnan(c.kv.v[0, free].float()).all()


def test_captured_and_replayed():
    c = Cache([300, 70], 2, 64, True, 12, layers=2).to_dev()
    keep, sink, recent = [100, 30], [4, 0], [16, 8]
    k0, v0, m0 = c.kv.k.clone(), c.kv.v.clone(), c.dm.clone()
    kept = torch.zeros(2, 2, 130, dtype=torch.int32, device="cuda")
    ws = W.workspace(W.wisp_kv_evict_workspace_size(c.model, c.desc))
    W.wisp_kv_evict(c.model, c.kv, c.desc, keep, c.dm, kept, ws, sink, recent)
    want = [t.clone() for t in (c.kv.k, c.kv.v, c.dm, kept)]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        W.wisp_kv_evict(c.model, c.kv, c.desc, keep, c.dm, kept, ws, sink, recent)
    for i in range(3):
        for t, x in ((c.kv.k, k0), (c.kv.v, v0), (c.dm, m0)):
            t.copy_(x)
        kept.fill_(-1)
        g.replay()
        torch.cuda.synchronize()
        W.wisp_check(ws)
        for t, x in zip((c.kv.k, c.kv.v, c.dm, kept), want):
            assert torch.equal(t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32),
                               x.view(torch.int16) if x.dtype == torch.bfloat16 else x.view(torch.int32)), i


def test_attention_after_an_eviction_is_the_kept_tokens_own():
    """The cache that is left is one of keep tokens at positions 0 .. keep - 1: wisp_attention and
    wisp_attention_shared over it are what fp64 makes of the kept keys at their new positions."""
    c = Cache([500, 123], 2, 64, False, 13)
    c.to_dev()
    keep = [100, 64]
    kept = c.run(keep, [4, 4], [30, 30])
    c.check(kept, keep, [4, 4], [30, 30])
    ctx = np.array(keep, np.int32) - 1                        # the last kept token stands for a new one
    desc = W.BatchDesc(ctx, np.zeros(2, np.int32), to_dev(c.pt))
    q = c.rng.normal(0, 1, (2, 2, 64)).astype(np.float32)
    out, lse = torch.empty(2, 2, 64, device="cuda"), torch.empty(2, 2, device="cuda")
    plan = W.wisp_shared_plan(c.model, desc, None, None, W.workspace(W.wisp_shared_workspace_size(c.model, desc)))
    W.wisp_attention_shared(plan, c.kv, to_dev(q), out, lse)
    ref, rl, _, _ = shared.attention(q.astype(np.float64), c.k[0], c.v[0], c.pt, ctx, [1, 1])
    np.testing.assert_allclose(out.cpu().numpy(), ref, atol=(2 * 72 * 20 + 400) * U * 3)
    np.testing.assert_allclose(lse.cpu().numpy(), rl, atol=(72 * 20 + 400) * U)
    old = torch.empty_like(out)
    W.wisp_attention(c.model, c.kv, desc, to_dev(q), old, W.workspace(W.wisp_workspace_size(c.model, desc)))
    np.testing.assert_allclose(old.cpu().numpy(), ref, atol=(2 * 72 * 20 + 400) * U * 3)
