"""Pins of the 8-bit cache's oracle on the CPU: its codes against torch's e4m3 type, its page
orders, its scales, and the host-side refusals of the entry points."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from kv8_harness import shape
from oracle import kv8

FAKE = 0x1000  # never dereferenced: validation fails first


def test_codes_are_e4m3():
    c = torch.arange(256, dtype=torch.uint8)
    np.testing.assert_array_equal(c.view(torch.float8_e4m3fn).double().numpy(), kv8.VALUES)
    x = np.concatenate([kv8.VALUES[:127], (kv8.VALUES[:126] + kv8.VALUES[1:127]) / 2, np.linspace(-448, 448, 4001), [np.nan, -0.0]])
    got = torch.from_numpy(x).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(got, kv8.e4m3_encode(x.astype(np.float32)))


@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
def test_page_orders_are_permutations(hd):
    for order in (kv8.k_order(hd), kv8.v_order(hd)):
        assert sorted(order.reshape(-1)) == list(range(16 * hd))


def test_scales_are_the_smallest_powers():
    for most, want in ((0.0, 1.0), (448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1e-45, 2.0 ** -100), (448 * 2.0 ** 100, 2.0 ** 100)):
        assert kv8.scale_of(most) == want


def test_append_in_steps_gives_the_page_of_one_step():
    """Rows appended one at a time: the same scale as at once, codes off by what the smaller
    scales before rounded."""
    rng = np.random.default_rng(5)
    n_kv, hd = 1, 32
    qkv = rng.normal(0, 1, (20, 3 * hd))
    pt = np.array([[0, 1]])
    one = [np.zeros((2, 1, 16 * hd), np.uint8) for _ in range(2)] + [np.ones((2, 1, 2))]
    many = [a.copy() for a in one]
    kv8.append(*one, pt, [0], [20], qkv, 1, 1, hd, 1e4)
    for t in range(20):
        kv8.append(*many, pt, [t], [1], qkv[t:t + 1], 1, 1, hd, 1e4)
    np.testing.assert_array_equal(one[2], many[2])
    a, b = (kv8.tokens(s[0], s[2], "k", pt[0], 0, 20, hd) for s in (one, many))
    assert np.all(np.abs(a - b) <= 2.0 ** -3 * np.abs(a) + 2.0 ** -9 * one[2].max())


# ----- refusals --------------------------------------------------------------------------
def _desc(ctx, gamma, stride=16, prefill=None):
    d = W.BatchDesc(ctx, gamma, None, 1.0, prefill_len=prefill)
    d.c.kv_page_table = FAKE
    d.c.pt_stride = stride
    return d


def _plan(model, desc, ws=FAKE, n=1 << 40):
    b = W.wisp_kv8_batch()
    return W.load_library().wisp_kv8_plan(C.byref(model), C.byref(desc.c), ws, n, C.byref(b), None)


def test_plan_refusals():
    m = W.GpuModel.shape_only(shape(8, 2, 64, True))
    assert W.wisp_kv8_workspace_size(m, _desc([10], [2])) > 256
    assert W.wisp_kv8_workspace_size(m, _desc([10], [17])) == 0
    assert W.wisp_kv8_workspace_size(W.GpuModel.shape_only(shape(8, 2, 96, True)), _desc([10], [2])) == 0
    assert W.wisp_kv8_workspace_size(W.GpuModel.shape_only(shape(8, 2, 96, False)), _desc([10], [2])) > 0
    assert W.wisp_kv8_workspace_size(W.GpuModel.shape_only(shape(8, 3, 64, True)), _desc([10], [2])) == 0
    assert _plan(m, _desc([-1], [2])) == W.WISP_E_INVALID
    assert _plan(m, _desc([250], [8])) == W.WISP_E_CAPACITY
    L = W.load_library()
    assert L.wisp_kv8_plan(C.byref(m), C.byref(_desc([1], [1]).c), FAKE, 1 << 40, None, None) == W.WISP_E_INVALID
    # a batch that would pass the work list's 2^22 items: every request one on each of 32 kv heads
    n = 1 << 17
    big = _desc([5] * n, [0] * n)
    assert W.wisp_kv8_workspace_size(W.GpuModel.shape_only(shape(32, 32, 64, True)), big) == 0
    assert "work items" in W.wisp_last_error()
    # one that would pass an append's 2^32 threads: prompts of 229 thousand rows on 2048 heads
    m = W.GpuModel.shape_only(shape(2048, 2048, 128, True))
    wide = W.BatchDesc(np.zeros(7, np.int32), np.zeros(7, np.int32), None, 1.0, None, np.full(7, 32768, np.int32))
    assert W.wisp_kv8_workspace_size(m, wide) == 0
    assert "threads" in W.wisp_last_error()
    # long contexts do not: 64 requests of 2^29 tokens
    ctx = 1 << 29
    far = _desc([ctx] * 64, [0] * 64, stride=(ctx >> 4) + 1)
    assert W.wisp_kv8_workspace_size(W.GpuModel.shape_only(shape(8, 8, 64, True)), far) > 0


def test_calls_need_a_planned_batch():
    L = W.load_library()
    b, kv = W.wisp_kv8_batch(), W.wisp_kv8(FAKE, FAKE, FAKE, 4, 16)
    assert L.wisp_attention_kv8(C.byref(b), C.byref(kv), FAKE, FAKE, None) == W.WISP_E_INVALID
    assert "planned" in W.wisp_last_error()
    assert L.wisp_kv8_append(C.byref(b), C.byref(kv), FAKE, 1 << 20, FAKE, None) == W.WISP_E_INVALID
    assert L.wisp_attention_kv8(None, C.byref(kv), FAKE, FAKE, None) == W.WISP_E_INVALID
    assert L.wisp_kv8_append(None, None, None, 0, None, None) == W.WISP_E_INVALID
