"""wisp_token_logprobs at the edges of its arguments: outputs left out, the smallest temperatures,
vocabularies and batches that take kernels of their own."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
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
