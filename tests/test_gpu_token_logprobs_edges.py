"""wisp_token_logprobs at the edges of its arguments: outputs left out, the smallest temperatures,
vocabularies and batches that take kernels of their own."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
import test_gpu_token_logprobs as base
from gpu_harness import log

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [0, 3])
def test_tokens_out_of_range_are_reported_without_their_log_probability(top):
    V = 1000
    x = torch.randn(3, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    H = torch.zeros(3, device="cuda")
    ids = torch.zeros(3, top, dtype=torch.int32, device="cuda") if top else None
    tlp = torch.zeros(3, top, device="cuda") if top else None
    for bad in (V, -2, 2 ** 31 - 1):
        log(f"entropy alone, top {top}, a token of {bad}")
        tok = torch.tensor([5, bad, -1], dtype=torch.int32, device="cuda")
        ws = W.workspace(W.wisp_token_logprobs_workspace_size(3, V, top))
        W.wisp_token_logprobs(x, V, tok, 1.0, None, H, ids, tlp, ws)
        with pytest.raises(W.WispError) as e:
            W.wisp_check(ws)
        assert e.value.status == W.WISP_E_DEVICE_INPUT
    ws = W.workspace(W.wisp_token_logprobs_workspace_size(3, V, top))
    W.wisp_token_logprobs(x, V, torch.tensor([5, 0, -1], dtype=torch.int32, device="cuda"), 1.0, None, H, ids, tlp, ws)
    W.wisp_token_logprobs(x, V, None, 1.0, None, H, ids, tlp, ws)
    W.wisp_check(ws)


@pytest.mark.parametrize("T", [1e-45, 1e-40, 4e-39, 5e-39, 1e-30, 1e38, 3.4e38])
@pytest.mark.parametrize("V", [1000, 20001])
def test_temperatures_at_the_ends_of_fp32(T, V):
    """Almost all of p on the largest logits, or all tokens alike."""
    T = float(np.float32(T))
    x = torch.randn(3, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(V))
    x[0, V - 7] = 9.0
    x[1, [3, V // 2]] = 9.0
    x[2] = x[2].clamp(max=1.0)                   # hundreds of the largest
    tok = torch.tensor([V - 7, V // 2, 0], dtype=torch.int32, device="cuda")
    lp, H = torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda")
    ids, tlp = torch.zeros(3, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, device="cuda")
    W.wisp_token_logprobs(x, V, tok, T, lp, H, ids, tlp, W.workspace(W.wisp_token_logprobs_workspace_size(3, V, 4)))
    z = x.double() / T
    d = z - z.amax(-1, keepdim=True)
    ls = d - torch.log(torch.exp(d).sum(-1, keepdim=True))
    want = (ls.gather(1, tok.long()[:, None])[:, 0], -(torch.exp(ls) * ls).sum(-1), torch.sort(ls, dim=-1, descending=True)[0][:, :4])
    log(f"T={T} V={V}: ln p {lp.tolist()}, entropy {H.tolist()}")
    for g, w in zip((lp, H, tlp), want):
        w32 = w.float()                          # -infinity below fp32's range
        assert not torch.isnan(g).any() and torch.equal(torch.isinf(g), torch.isinf(w32))
        fin = ~torch.isinf(w32)
        # a chunk's exponentials and sums: 2^-22 of 16 binary orders each, and the result's rounding
        assert ((g.double() - w).abs()[fin] <= 2.0 ** -23 * w.abs()[fin] + 2.0 ** -17).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(7, 0), (0, 1)], ids=["wide loads", "single loads"])
def test_vocabularies_of_more_chunks_than_a_thread_holds(pad, shift, dtype):
    V = 270001
    low = torch.finfo(dtype).min
    x, tok = base._logits(6, V, dtype, 21, pad, shift)
    x[1, :V] = low                              # a mask's lowest value: too many to rank at once
    x[1, [V // 3, V - 1, 5]] = torch.tensor([1.0, 1.0, -2.0], device="cuda", dtype=dtype)
    x[2, :V] = -float("inf")
    x[3, :V] = 0.0
    x[4, V - 1] = 30.0                          # the last entry of the last chunk
    tok[1], tok[4] = 5, V - 1
    for top in (0, 1, 32):
        got, ws = base._run(x, V, tok, 1.0, top)
        W.wisp_check(ws)
        log(f"  top {top}: worst {base._check(x, V, tok, 1.0, top, got):.3f} of its bound")


def test_most_probable_tokens_of_more_rows_than_a_launch_takes():
    rows, V, top = (1 << 23) + 261, 2, 1
    x = torch.randn(rows, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    tok = torch.arange(rows, device="cuda", dtype=torch.int32) % 3 - 1       # every third row has none
    lp, H = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
    ids, tlp = torch.full((rows, top), 7, dtype=torch.int32, device="cuda"), torch.full((rows, top), 7.0, device="cuda")
    ws = W.workspace(W.wisp_token_logprobs_workspace_size(rows, V, top))
    log(f"{rows} rows, {ws.numel() >> 20} MB of workspace")
    W.wisp_token_logprobs(x, V, tok, 1.0, lp, H, ids, tlp, ws)
    W.wisp_check(ws)
    on, ls = tok >= 0, torch.log_softmax(x.double(), -1)
    first = x[:, 1] > x[:, 0]
    assert torch.equal(ids[on, 0], first[on].int())
    # two entries: a handful of fp32 roundings of terms below 16
    for g, w in ((lp, ls.gather(1, tok.clamp_min(0).long()[:, None])[:, 0]), (tlp[:, 0], ls.amax(-1)), (H, -(ls.exp() * ls).sum(-1))):
        assert ((g.double() - w).abs()[on] <= 64 * 2.0 ** -24 * (1 + w.abs()[on])).all()
        assert (g[~on] == 7).all()
    assert (ids[~on] == 7).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 7, 8193, 50257, 270001])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_a_single_row_of_any_length(shift, V, dtype):
    """Its length says nothing of its start: wide loads where that is on 16 bytes, up to the last entry."""
    x, tok = base._logits(1, V, dtype, 31 + V, 0, shift)
    x[0, V - 1] = 12.0
    tok[0] = V - 1
    for top in (0, 5):
        got, ws = base._run(x, V, tok, 1.0, top)
        W.wisp_check(ws)
        log(f"one row of {V}, off by {shift}, top {top}: worst {base._check(x, V, tok, 1.0, top, got):.3f} of its bound")
