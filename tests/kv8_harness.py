"""Shared set-up of the 8-bit cache's tests: seeded caches and batches on both sides."""
from __future__ import annotations

import numpy as np
import torch

import paper_2601_11652_amd as W
import wisp_inputs as wi
from gpu_harness import to_dev
from oracle import kv8


def shape(n_q, n_kv, hd, bf16, base=1e4):
    return wi.ModelShape("kv8", 1, 256, n_q, n_kv, hd, 256, 256, "bf16" if bf16 else "f32", base)


def round_to(a: np.ndarray, bf16: bool) -> np.ndarray:
    """fp64 values of a rounded to the storage type."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return (t.to(torch.bfloat16) if bf16 else t).double().numpy()


def dev(a: np.ndarray, bf16: bool) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16 if bf16 else torch.float32).cuda()


class Case:
    """A batch over a scattered, seeded cache.  Every slot past a request's cached tokens, and every
    page that no request uses, holds NaN codes (V too) and a NaN scale where no append has to read
    it."""

    def __init__(self, ctx, nrow, n_q, n_kv, hd, bf16, seed, base=1e4, pow2=True, gamma=None):
        self.rng = rng = np.random.default_rng(seed)
        self.ctx, self.nrow = np.asarray(ctx, np.int32), np.asarray(nrow, np.int32)
        self.n_q, self.n_kv, self.hd, self.bf16, self.base = n_q, n_kv, hd, bf16, base
        self.gamma = np.minimum(self.nrow - 1, 16) if gamma is None else np.asarray(gamma, np.int32)
        pre = self.nrow - 1 - self.gamma
        self.shape = shape(n_q, n_kv, hd, bf16, base)
        self.model = W.GpuModel.shape_only(self.shape)
        need = (self.ctx + self.nrow + 15) // 16
        nb = int(need.sum()) + 4
        perm = rng.permutation(nb).astype(np.int32)
        self.pt = np.full((len(self.ctx), int(need.max()) + 2), -1, np.int32)
        self.k = np.full((nb, n_kv, 16 * hd), kv8.NAN_CODE, np.uint8)
        self.v = self.k.copy()
        self.scale = np.full((nb, n_kv, 2), np.nan, np.float32)
        ko, vo = kv8.k_order(hd), kv8.v_order(hd)
        o = 0
        for b in range(len(self.ctx)):
            self.pt[b, :need[b]] = perm[o:o + need[b]]
            for p in range(need[b]):
                blk, held = self.pt[b, p], min(max(int(self.ctx[b]) - 16 * p, 0), 16)
                for pool, order in ((self.k, ko), (self.v, vo)):
                    page = pool[blk].copy()
                    codes = kv8.e4m3_encode(np.clip(rng.normal(0, 90, (n_kv, held, hd)), -448, 448))
                    page[:, order[:held].reshape(-1)] = codes.reshape(n_kv, -1)
                    pool[blk] = page
                sc = 2.0 ** rng.integers(-8, -4, (n_kv, 2)) if pow2 else rng.uniform(0.004, 0.05, (n_kv, 2))
                if held:
                    self.scale[blk] = sc
            o += int(need[b])
        self.M = int(self.nrow.sum())
        self.desc = W.BatchDesc(self.ctx, self.gamma, to_dev(self.pt) if torch.cuda.is_available() else None, 1.0, None,
                                pre if pre.any() else None)

    def pool(self) -> W.KV8Pool:
        f8 = lambda a: torch.from_numpy(a.copy())[None].cuda().view(torch.float8_e4m3fn)
        return W.KV8Pool(f8(self.k), f8(self.v), torch.from_numpy(self.scale.copy())[None].cuda())

    def plan(self, stream=None) -> W.KV8Batch:
        return W.wisp_kv8_plan(self.model, self.desc, W.workspace(W.wisp_kv8_workspace_size(self.model, self.desc)), stream)

    def qkv(self, std=1.15) -> np.ndarray:
        return round_to(self.rng.normal(0, std, (self.M, (self.n_q + 2 * self.n_kv) * self.hd)), self.bf16)

    def queries(self, std=1.15) -> np.ndarray:
        return round_to(self.rng.normal(0, std, (self.M, self.n_q, self.hd)), self.bf16)

    def fill(self):
        """Gives the new rows' slots codes too, as an append would: attention alone."""
        ko, vo = kv8.k_order(self.hd), kv8.v_order(self.hd)
        for b in range(len(self.ctx)):
            end = int(self.ctx[b] + self.nrow[b])
            for p in range(int(self.ctx[b]) // 16, (end + 15) // 16):
                blk, a, e = self.pt[b, p], max(int(self.ctx[b]) - 16 * p, 0), min(end - 16 * p, 16)
                for pool, order in ((self.k, ko), (self.v, vo)):
                    page = pool[blk].copy()
                    page[:, order[a:e].reshape(-1)] = kv8.e4m3_encode(
                        np.clip(self.rng.normal(0, 90, (self.n_kv, e - a, self.hd)), -448, 448)).reshape(self.n_kv, -1)
                    pool[blk] = page
                if a == 0:
                    self.scale[blk] = 2.0 ** self.rng.integers(-8, -4, (self.n_kv, 2))
        return self


def host_pool(kv: W.KV8Pool):
    return (kv.k[0].view(torch.uint8).cpu().numpy().copy(), kv.v[0].view(torch.uint8).cpu().numpy().copy(),
            kv.scale[0].cpu().numpy().astype(np.float64))


def attention_bound(ref, mag, big, hd, T, bf16):
    """What separates a result from fp64's.  Scores: the sum of hd products in fp32, off by at most
    hd half steps (2^-24) of the terms' magnitude, and of the scale and the exponential 8 more.
    bf16: a probability is rounded once (2^-8), in numerator and sum, and the output (2^-8).  fp32:
    the sums over T tokens, and three roundings."""
    d = (hd + 8) * 2.0 ** -24 * np.maximum(big, 1.0)[..., None]
    sums = (T + 16) * 2.0 ** -24
    if bf16:
        return 2.0 ** -8 * np.abs(ref) + (2 * 2.0 ** -8 + 2 * d + 2 * sums) * mag
    return (2 * d + 2 * sums) * mag + 2.0 ** -24 * np.abs(ref)
