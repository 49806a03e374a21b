"""Host-side refusals of the operators on shared prefixes and of the eviction, before any GPU work."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_11652_amd as W
from fake_device import Calls, fake
from shared_harness import shape

FAKE = 0x10000  # never dereferenced: validation fails first


def _model(n_q=8, n_kv=2, hd=64, bf16=True, layers=1):
    return W.GpuModel.shape_only(shape(n_q, n_kv, hd, bf16, layers))


def _desc(ctx, gamma=None, prefill=None, stride=64, table=FAKE):
    d = W.BatchDesc(ctx, np.zeros(len(ctx), np.int32) if gamma is None else gamma, None, 1.0, prefill_len=prefill)
    d.c.kv_page_table, d.c.pt_stride = table, stride
    return d


def _plan(model, desc, size, prefix, ws=FAKE, nbytes=1 << 40, batch=None):
    n, ps, pp, _keep = W._groups(size, prefix)
    b = W.wisp_shared_batch() if batch is None else batch
    return W.load_library().wisp_shared_plan(C.byref(model), C.byref(desc.c), n, ps, pp, ws, nbytes, C.byref(b), None)


@pytest.mark.parametrize("size,prefix,why", [
    ([2, 2], [16, 0], "add up"),            # B is 3
    ([2], [16], "add up"),
    ([0, 3], [16, 16], "positive"),
    ([-1, 4], [0, 0], "positive"),
    ([2 ** 31 - 1], [0], "positive"),
    ([3], [8], "whole pages"),
    ([3], [-16], "whole pages"),
    ([2, 1], [48, 16], "cached tokens"),    # request 1 has 40
    ([2, 1], [16, 64], "cached tokens"),
])
def test_groups(size, prefix, why):
    m, d = _model(), _desc([100, 40, 50])
    assert _plan(m, d, size, prefix) == W.WISP_E_INVALID
    assert why in W.wisp_last_error()
    assert W.wisp_shared_workspace_size(m, d, size, prefix) == 0


def test_group_arrays():
    m, d = _model(), _desc([100, 40, 50])
    L, b = W.load_library(), W.wisp_shared_batch()
    one = (C.c_int32 * 1)(3)
    for n, s, p in ((-1, one, one), (1, None, one), (1, one, None)):
        assert L.wisp_shared_plan(C.byref(m), C.byref(d.c), n, s, p, FAKE, 1 << 40, C.byref(b), None) == W.WISP_E_INVALID
    with pytest.raises(ValueError):
        W.wisp_shared_workspace_size(m, d, [3], None)
    with pytest.raises(ValueError):
        W.wisp_shared_workspace_size(m, d, [2, 1], [16])


def test_workspaces_and_tables():
    m, d = _model(), _desc([100, 40, 50])
    need = W.wisp_shared_workspace_size(m, d, [3], [32])
    assert need > 256 and W.wisp_shared_workspace_size(m, d) > 256
    assert _plan(m, d, [3], [32], nbytes=need - 1) == W.WISP_E_WORKSPACE
    assert _plan(m, d, [3], [32], ws=FAKE + 128) == W.WISP_E_INVALID
    assert _plan(m, d, [3], [32], ws=None) == W.WISP_E_INVALID
    assert _plan(m, _desc([100, 40, 50], stride=6), [3], [32]) == W.WISP_E_CAPACITY
    assert _plan(m, _desc([100, 40, 50], table=None), [3], [32]) == W.WISP_E_INVALID
    assert W.load_library().wisp_shared_plan(C.byref(m), C.byref(d.c), 0, None, None, FAKE, need, None, None) == W.WISP_E_INVALID


def test_sizes_beyond_the_kernels():
    assert W.wisp_shared_workspace_size(_model(65, 1, 64, False), _desc([5])) == 0            # more than 64 query heads per kv head
    assert W.wisp_shared_workspace_size(_model(64, 1, 64, False), _desc([5])) > 0
    assert W.wisp_shared_workspace_size(_model(1 << 16, 1 << 16, 32, False), _desc([5])) == 0  # more than 65535 kv heads
    assert W.wisp_shared_workspace_size(_model(65535, 65535, 32, False), _desc([5])) > 0
    assert W.wisp_shared_workspace_size(_model(32768, 1024, 128), _desc([5])) > 0
    assert W.wisp_shared_workspace_size(_model(32768 + 32, 1024 + 1, 128), _desc([5])) == 0    # more than 2^22 values of q in a row
    rows = [32768] * 8
    assert W.wisp_shared_workspace_size(_model(), _desc([0] * 8, prefill=rows)) == 0           # more than WISP_ROWS_MAX rows
    # 2^30 - 1 tokens: more blocks of them than work items
    assert _plan(_model(), _desc([2 ** 30 - 17], stride=2 ** 27), None, None) == W.WISP_E_UNSUPPORTED
    assert W.wisp_shared_workspace_size(_model(), _desc([2 ** 27], stride=2 ** 24)) > 0


def test_calls_on_a_batch_that_was_not_planned():
    L, b, kv = W.load_library(), W.wisp_shared_batch(), W.wisp_kv(FAKE, FAKE, 4, 16)
    for batch in (None, C.byref(b)):
        assert L.wisp_attention_shared(batch, C.byref(kv), FAKE, FAKE, FAKE, None) == W.WISP_E_INVALID
        assert L.wisp_attention_mass(batch, C.byref(kv), FAKE, FAKE, None, 1.0, None, FAKE, None) == W.WISP_E_INVALID
    # one whose plan failed
    assert _plan(_model(), _desc([100]), [1], [7], batch=b) == W.WISP_E_INVALID
    assert L.wisp_attention_shared(C.byref(b), C.byref(kv), FAKE, FAKE, FAKE, None) == W.WISP_E_INVALID


def _evict(model=None, desc=None, keep=(10,), sink=None, recent=None, to=None, stride=0, mass=FAKE, kept=FAKE, ws=FAKE, nbytes=1 << 30,
           kv=None):
    model, desc = model or _model(), desc or _desc([100])
    (ka, k), (sa, s), (ra, r) = (W._host_i32(x, "x") for x in (keep, sink, recent))
    kv = kv or W.wisp_kv(FAKE, FAKE, 4, 16)
    return W.load_library().wisp_kv_evict(C.byref(model), C.byref(kv), C.byref(desc.c), k, s, r, to, stride, mass, kept, ws, nbytes, None)


@pytest.mark.parametrize("args,status", [
    (dict(keep=[-1]), W.WISP_E_INVALID),
    (dict(keep=None), W.WISP_E_INVALID),
    (dict(sink=[-1]), W.WISP_E_INVALID),
    (dict(recent=[-2]), W.WISP_E_INVALID),
    (dict(sink=[6], recent=[5]), W.WISP_E_INVALID),
    (dict(sink=[2 ** 31 - 1], recent=[2 ** 31 - 1]), W.WISP_E_INVALID),
    (dict(mass=None), W.WISP_E_INVALID),
    (dict(kept=None), W.WISP_E_INVALID),
    (dict(ws=None), W.WISP_E_INVALID),
    (dict(ws=FAKE + 16), W.WISP_E_INVALID),
    (dict(nbytes=256), W.WISP_E_WORKSPACE),
    (dict(to=FAKE, stride=0), W.WISP_E_CAPACITY),
    (dict(desc=_desc([100], stride=6)), W.WISP_E_CAPACITY),
    (dict(desc=_desc([100], table=None)), W.WISP_E_INVALID),
    (dict(desc=_desc([-1])), W.WISP_E_INVALID),
    (dict(desc=_desc([2 ** 30], stride=2 ** 27)), W.WISP_E_INVALID),
    (dict(kv=W.wisp_kv(None, FAKE, 4, 16)), W.WISP_E_INVALID),
    (dict(kv=W.wisp_kv(FAKE, FAKE + 8, 4, 16)), W.WISP_E_INVALID),
    (dict(kv=W.wisp_kv(FAKE, FAKE, 0, 16)), W.WISP_E_INVALID),
    (dict(kv=W.wisp_kv(FAKE, FAKE, 4, 32)), W.WISP_E_UNSUPPORTED),
    (dict(model=_model(hd=96)), W.WISP_E_UNSUPPORTED),
    (dict(desc=_desc([2 ** 30 - 1] * 3, stride=2 ** 26), keep=[2 ** 30 - 2] * 3), W.WISP_E_UNSUPPORTED),
])
def test_evictions(args, status):
    assert _evict(**args) == status, W.wisp_last_error()


@pytest.mark.parametrize("model,n,blocks", [
    (_model(8, 8, 128), 1 << 16, 4),                         # 2^22 workgroups of 1024 threads
    (_model(1 << 17, 1 << 17, 64), 1, 4),                    # kv heads
    (_model(8, 8, 64), 1, 1 << 24),                          # places in a pool
])
def test_evictions_beyond_the_kernels(model, n, blocks):
    call = lambda n, blocks: _evict(model, _desc([2] * n), [1] * n, kv=W.wisp_kv(FAKE, FAKE, blocks, 16), nbytes=256)
    assert call(n, blocks) == W.WISP_E_UNSUPPORTED, W.wisp_last_error()
    if model.n_kv_heads <= 65535:                            # one less is refused for its workspace only
        assert call(max(n - 1, 1), min(blocks, (1 << 24) - 1)) == W.WISP_E_WORKSPACE


def test_evictions_of_nothing():
    """No request, or none that keeps a token: nothing to do, and no pointer is needed."""
    assert _evict(desc=_desc([], table=None), keep=[], mass=None, kept=None, ws=None) == W.WISP_OK
    assert _evict(keep=[0], kept=None) == W.WISP_OK
    assert W.wisp_kv_evict_workspace_size(_model(), _desc([])) == 256


# the binding: devices, types and sizes are refused before the library sees a pointer
NAMES = ("kv", "q", "out", "lse", "prev", "mass", "count")


def _batch(index=0):
    d = W.BatchDesc(np.array([20, 20]), np.array([2, 0]), fake(2, 2, dtype=torch.int32, index=index), 1.0)
    return W.wisp_shared_plan(_model(4, 2, 32, False), d, [2], [16], fake(4096, dtype=torch.uint8, index=index))


def _calls(at, plan):
    i = lambda n: at.get(n, 0)
    kv = W.KVPool(fake(1, 4, 2, 16 * 32, index=i("kv")), fake(1, 4, 2, 16 * 32, index=i("kv")))
    q, lse = fake(4, 4, 32, index=i("q")), fake(4, 4, index=i("lse"))
    yield "shared", lambda: W.wisp_attention_shared(plan, kv, q, fake(4, 4, 32, index=i("out")), lse)
    yield "mass", lambda: W.wisp_attention_mass(plan, kv, q, lse, fake(4, 2, 16, index=i("mass")), fake(4, 2, 16, index=i("prev")), 1.0,
                                                fake(2, dtype=torch.int32, index=i("count")))


def test_calls_run_on_their_tensors_device(monkeypatch):
    c = Calls(monkeypatch)
    plan = _batch(1)
    for _, f in _calls({n: 1 for n in NAMES}, plan):
        f()
    assert [(n, on) for (n, _), on in zip(c.calls, c.devices)] == [("wisp_shared_plan", 1), ("wisp_attention_shared", 1), ("wisp_attention_mass", 1)]
    assert c.on == 0


@pytest.mark.parametrize("name", NAMES)
def test_calls_refuse_a_second_device(monkeypatch, name):
    c = Calls(monkeypatch)
    plan = _batch()
    refused = 0
    for _, f in _calls({name: 1}, plan):
        try:
            f()
        except ValueError:
            refused += 1
    assert refused == (1 if name in ("out", "prev", "mass", "count") else 2)
    assert len(c.calls) == 3 - refused


def test_plan_refuses_a_table_of_another_device(monkeypatch):
    c = Calls(monkeypatch)
    d = W.BatchDesc(np.array([20]), np.array([2]), fake(1, 2, dtype=torch.int32, index=1), 1.0)
    with pytest.raises(ValueError):
        W.wisp_shared_plan(_model(), d, None, None, fake(4096, dtype=torch.uint8))
    assert not c.calls


def _evict_call(at=None, **kw):
    i = lambda n: (at or {}).get(n, 0)
    kv = W.KVPool(fake(2, 4, 2, 16 * 64, dtype=torch.bfloat16, index=i("kv")), fake(2, 4, 2, 16 * 64, dtype=torch.bfloat16, index=i("kv")))
    d = W.BatchDesc(np.array([20, 9]), np.zeros(2, np.int32), fake(2, 2, dtype=torch.int32, index=i("page_table")), 1.0)
    a = dict(keep=[10, 9], mass=fake(2, 4, 2, 16, index=i("mass")), kept=fake(2, 2, 19, dtype=torch.int32, index=i("kept")),
             workspace=fake(4096, dtype=torch.uint8, index=i("workspace")), to_table=fake(2, 1, dtype=torch.int32, index=i("to_table")))
    a.update(kw)
    W.wisp_kv_evict(_model(layers=2), kv, d, **a)


def test_eviction_runs_on_its_tensors_device(monkeypatch):
    c = Calls(monkeypatch)
    _evict_call({n: 1 for n in ("kv", "page_table", "mass", "kept", "workspace", "to_table")})
    assert c.calls[-1][0] == "wisp_kv_evict" and c.devices == [1]


@pytest.mark.parametrize("name", ["kv", "page_table", "mass", "kept", "workspace", "to_table"])
def test_eviction_refuses_a_second_device(monkeypatch, name):
    c = Calls(monkeypatch)
    with pytest.raises(ValueError):
        _evict_call({name: 1})
    assert not c.calls


@pytest.mark.parametrize("kw", [dict(kept=None), dict(keep=[10]), dict(sink=[1]), dict(recent=[1, 2, 3]), dict(keep=None)])
def test_eviction_refuses_sizes(monkeypatch, kw):
    c = Calls(monkeypatch)
    if kw.get("kept", 0) is None:
        kw = dict(kept=fake(2, 2, 18, dtype=torch.int32))
    with pytest.raises(ValueError):
        _evict_call(**kw)
    assert not c.calls
