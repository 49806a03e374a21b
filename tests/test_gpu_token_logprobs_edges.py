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
