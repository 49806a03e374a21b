"""The workspace that a call makes for itself belongs to the stream that the call runs on: made there,
it is cleared before the kernels and handed on only behind them."""
import pytest
import torch

import paper_2601_11652_amd as W
from fake_device import Calls, FakeStream, fake

STREAMS = [(None, 1), (FakeStream(7), 7), (9, 9), (0, 0)]


@pytest.mark.parametrize("stream,handle", STREAMS)
def test_token_logprobs_makes_its_workspace_on_its_stream(monkeypatch, stream, handle):
    c = Calls(monkeypatch)
    W.wisp_token_logprobs(fake(3, 100), 100, fake(3, dtype=torch.int32), 1.0, fake(3), stream=stream)
    name, args = c.calls[-1]
    assert name == "wisp_token_logprobs" and args[-1] == handle
    assert c.made == [(4096, handle)] and c.current == 1


@pytest.mark.parametrize("stream,handle", STREAMS)
def test_draft_stats_makes_its_workspace_on_its_stream(monkeypatch, stream, handle):
    c = Calls(monkeypatch)
    W.wisp_draft_stats(fake(3, 100), 100, 1.0, fake(3, 4), stream=stream)
    name, args = c.calls[-1]
    assert name == "wisp_draft_stats" and args[-1] == handle
    assert c.made == [(4096, handle)] and c.current == 1
