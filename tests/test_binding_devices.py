"""Calls whose tensors are on several devices are refused before the library sees a pointer."""
import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
import wisp_inputs as wi
from fake_device import Calls, fake

SHAPE = wi.ModelShape("two", 2, 64, 4, 2, 32, 64, 96, "f32", 1e4)


def _step(**on):
    """One verification step on the 8-bit cache, its tensors on device 0 but for those named."""
    at = lambda name: on.get(name, 0)
    f8, i32 = torch.float8_e4m3fn, torch.int32
    kv = W.KV8Pool(*(fake(2, 4, 2, 16 * 32, dtype=f8, index=at("kv")) for _ in range(2)),
                   fake(2, 4, 2, 2, index=at("kv")))
    desc = W.BatchDesc(np.array([3]), np.array([2]), fake(1, 2, dtype=i32, index=at("page_table")), 1.0)
    W.wisp_verify_kv8(W.GpuModel.shape_only(SHAPE), kv, desc, fake(3, dtype=i32, index=at("tokens")),
                      fake(2, 96, index=at("draft_probs")), 1, fake(1, dtype=i32, index=at("accept_len")),
                      fake(3, dtype=i32, index=at("out_tokens")), fake(3, 96, index=at("target_logits")),
                      fake(4096, dtype=torch.uint8, index=at("workspace")))


def test_one_device_is_taken(monkeypatch):
    c = Calls(monkeypatch)
    _step()
    assert c.calls[-1][0] == "wisp_verify_kv8"


@pytest.mark.parametrize("name", ["tokens", "draft_probs", "accept_len", "out_tokens", "target_logits", "workspace", "page_table", "kv"])
def test_the_step_refuses_a_second_device(monkeypatch, name):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        _step(**{name: 1})
    assert not c.calls


def test_calls_run_on_their_tensors_device(monkeypatch):
    c = Calls(monkeypatch)
    W.wisp_draft_stats(fake(3, 100, index=1), 100, 1.0, fake(3, 4, index=1))
    W.wisp_token_logprobs(fake(3, 100, index=1), 100, fake(3, dtype=torch.int32, index=1), 1.0, fake(3, index=1))
    _step(**{n: 1 for n in ("tokens", "draft_probs", "accept_len", "out_tokens", "target_logits", "workspace", "page_table", "kv")})
    ran = {name: on for (name, _), on in zip(c.calls, c.devices) if not name.endswith("_size")}
    assert ran == {"wisp_draft_stats": 1, "wisp_token_logprobs": 1, "wisp_verify_kv8": 1}
    assert c.on == 0


@pytest.mark.parametrize("name", ["stats", "ws"])
def test_draft_stats_refuses_a_second_device(monkeypatch, name):
    c = Calls(monkeypatch)
    at = {name: 1}
    with pytest.raises(ValueError):
        W.wisp_draft_stats(fake(3, 100), 100, 1.0, fake(3, 4, index=at.get("stats", 0)),
                           fake(4096, dtype=torch.uint8, index=at.get("ws", 0)))
    assert not c.calls
