"""Host-side refusals of the step on the 8-bit cache, before any GPU work."""
import ctypes as C

import numpy as np
import pytest

import paper_2601_11652_amd as W
from kv8_harness import shape

FAKE = 0x10000  # never dereferenced: validation fails first


def _step(ws, model=None):
    m = model or W.GpuModel.shape_only(shape(8, 2, 64, True))
    ptrs = (C.c_void_p * 1)(FAKE)
    m.embed = m.final_norm = m.lm_head = FAKE
    for name in ("attn_norm", "w_qkv", "w_o", "mlp_norm", "w_gate_up", "w_down"):
        setattr(m, name, C.cast(ptrs, dict(m._fields_)[name]))
    d = W.BatchDesc(np.array([10]), np.array([2]), None, 1.0)
    d.c.kv_page_table, d.c.pt_stride = FAKE, 4
    kv = W.wisp_kv8(FAKE, FAKE, FAKE, 4, 16)
    # a workspace too small by any measure: the last refusal before the GPU
    return W.load_library().wisp_verify_kv8(C.byref(m), C.byref(kv), C.byref(d.c), FAKE, FAKE, 1, FAKE, FAKE, FAKE, ws, 256, None)


@pytest.mark.parametrize("off", [1, 2, 4, 8])
def test_workspaces_off_16_bytes(off):
    assert _step(FAKE + off) == W.WISP_E_INVALID
    assert "aligned" in W.wisp_last_error()
    assert _step(None) == W.WISP_E_INVALID


def test_aligned_workspaces_pass_that_check():
    for ws in (FAKE, FAKE + 16):
        assert _step(ws) == W.WISP_E_WORKSPACE
