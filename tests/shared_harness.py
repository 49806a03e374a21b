"""Shared set-up of the tests on caches whose prefixes requests share: seeded caches and batches."""
from __future__ import annotations

import numpy as np
import torch

import paper_2601_11652_amd as W
import wisp_inputs as wi
from gpu_harness import to_dev

U = 2.0 ** -24          # half a step of fp32
HALF = {True: 2.0 ** -8, False: U}   # of the storage type, by whether it is bf16


def shape(n_q, n_kv, hd, bf16, layers=1, base=1e4):
    return wi.ModelShape("shared", layers, 256, n_q, n_kv, hd, 256, 256, "bf16" if bf16 else "f32", base)


def torch_type(bf16):
    return torch.bfloat16 if bf16 else torch.float32


def to_pages(a: np.ndarray, which: str, bf16: bool) -> torch.Tensor:
    """Slot-major fp64 pages [..., 16, hd] -> device pages in the library's layout."""
    return wi.pages_from_slots(torch.from_numpy(np.ascontiguousarray(a)).to(torch_type(bf16)), which).cuda()


def from_pages(t: torch.Tensor, which: str, hd: int) -> torch.Tensor:
    """Device pages -> slot-major host pages [..., 16, hd] of the storage type."""
    return wi.slots_from_pages(t.cpu(), which, hd)


def bits(t: torch.Tensor) -> np.ndarray:
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).numpy()


class Case:
    """Groups of requests over a scattered cache: `groups` a list of (prefix, [(own cached tokens, rows),
    ...]).  Slots that no request has, and pages of none, hold NaN."""

    def __init__(self, groups, n_q, n_kv, hd, bf16, seed, std=1.15, spare=3):
        self.rng = rng = np.random.default_rng(seed)
        self.n_q, self.n_kv, self.hd, self.bf16 = n_q, n_kv, hd, bf16
        self.size = np.array([len(m) for _, m in groups], np.int32)
        self.prefix = np.array([p for p, _ in groups], np.int32)
        own = [m for _, ms in groups for m in ms]
        pre = np.repeat(self.prefix, self.size)
        self.ctx = np.array([c for c, _ in own], np.int32) + pre
        self.nrow = np.array([r for _, r in own], np.int32)
        self.gamma = np.minimum(self.nrow - 1, 16).astype(np.int32)
        prompt = self.nrow - 1 - self.gamma
        end = self.ctx + self.nrow
        tail = (end - pre + 15) // 16
        nb = int(tail.sum() + (self.prefix // 16).sum()) + spare
        perm = rng.permutation(nb).astype(np.int32)
        self.pt = np.full((len(own), int((end.max() + 15) // 16) + 2), -1, np.int32)
        self.k = np.full((nb, n_kv, 16, hd), np.nan)
        self.v = self.k.copy()
        o = i = 0
        fill = lambda n: self.round(rng.normal(0, std, (n, n_kv, 16, hd)))
        for p, ms in groups:
            common = perm[o:o + p // 16]
            o += p // 16
            self.k[common], self.v[common] = fill(p // 16), fill(p // 16)
            for _ in ms:
                blk = perm[o:o + tail[i]]
                o += int(tail[i])
                self.pt[i, :p // 16], self.pt[i, p // 16:p // 16 + tail[i]] = common, blk
                self.k[blk], self.v[blk] = fill(tail[i]), fill(tail[i])
                if end[i] % 16:
                    self.k[blk[-1], :, end[i] % 16:] = np.nan
                    self.v[blk[-1], :, end[i] % 16:] = np.nan
                i += 1
        self.M = int(self.nrow.sum())
        self.off = np.concatenate([[0], np.cumsum(self.nrow)])
        self.q = self.round(rng.normal(0, std, (self.M, n_q, hd)))
        self.model = W.GpuModel.shape_only(shape(n_q, n_kv, hd, bf16))
        self.desc = W.BatchDesc(self.ctx, self.gamma, to_dev(self.pt) if torch.cuda.is_available() else None, 1.0, None,
                                prompt if prompt.any() else None)

    def round(self, a):
        """To the storage type."""
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch_type(self.bf16)).double().numpy()

    def pool(self) -> W.KVPool:
        return W.KVPool(to_pages(self.k, "k", self.bf16)[None], to_pages(self.v, "v", self.bf16)[None])

    def plan(self, size=None, prefix=None, stream=None) -> W.SharedBatch:
        size, prefix = (self.size, self.prefix) if size is None else (size, prefix)
        ws = W.workspace(W.wisp_shared_workspace_size(self.model, self.desc, size, prefix))
        return W.wisp_shared_plan(self.model, self.desc, size, prefix, ws, stream)

    def alone(self):
        """The same batch with nothing shared."""
        return np.ones(len(self.ctx), np.int32), np.zeros(len(self.ctx), np.int32)

    def dev_q(self):
        return torch.from_numpy(self.q).to(torch_type(self.bf16)).cuda()

    def run(self, kv=None, plan=None, q=None, lse=True):
        """(out, lse) on the host, in fp64."""
        kv, plan = kv or self.pool(), plan or self.plan()
        out = torch.full((self.M, self.n_q, self.hd), float("nan"), dtype=torch_type(self.bf16), device="cuda")
        l = torch.full((self.M, self.n_q), float("nan"), device="cuda") if lse else None
        W.wisp_attention_shared(plan, kv, self.dev_q() if q is None else q, out, l)
        W.wisp_check(plan.ws)
        return out.double().cpu().numpy(), l.double().cpu().numpy() if lse else None


def attention_bounds(ref, lse, mag, big, hd, T, bf16):
    """What separates out and lse from fp64's.  A score is a sum of hd products in fp32, off by at most
    hd half steps of the terms' magnitude, and its scale, the difference from the maximum and the exponential add 8
    more: a probability is off by d of itself.  Sums over T tokens in some order, joined from parts of which
    each brings 4 roundings (fewer than 64 here), are off by `sums`.  bf16: a probability is rounded once before
    it multiplies V, and the output once."""
    d = (hd + 8) * U * np.maximum(big, 1.0)
    sums = (T + 256) * U
    out = HALF[bf16] * np.abs(ref) + ((HALF[True] if bf16 else 0.0) + 2 * d + 2 * sums)[..., None] * mag * (1 + HALF[bf16]) + 2 * U * np.abs(ref)
    return out, d + sums + 4 * U * np.maximum(np.abs(lse), 1.0)


def mass_bound(ref, err, got, prev, hd, rows):
    """A weight's exponent is off by (hd + 8) half steps of the score's terms and 4 of lse; the sum over
    `rows` rows, in 64 lanes and parts, by rows + 64; the decayed old weight by 2."""
    return (hd + 8) * U * (err + got) + (rows + 64) * U * got + 3 * U * np.abs(ref) + 2 * U * np.abs(prev)
