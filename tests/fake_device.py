"""Stand-ins for device tensors, streams and the library: what the Python binding does before a
call can be seen on the CPU."""
from __future__ import annotations

import contextlib

import torch

import paper_2601_11652_amd as W


class FakeTensor(torch.Tensor):
    """A host tensor that says it is on device `index`; nothing may run on it."""
    is_cuda = True
    index = 0

    @property
    def device(self):
        return torch.device("cuda", self.index)

    def get_device(self):
        return self.index


def fake(*shape, dtype=torch.float32, index=0):
    t = torch.Tensor._make_subclass(FakeTensor, torch.zeros(*shape, dtype=dtype))
    t.index = index
    return t


class FakeStream:
    def __init__(self, handle):
        self.cuda_stream = handle


class Calls:
    """Patches torch.cuda and the library.  `made`: (bytes, handle of the stream that was current) of
    every workspace; `calls`, `devices`: (name, arguments) of every library call, and the device current in it."""

    def __init__(self, monkeypatch, workspace_bytes=4096):
        self.made, self.calls, self.current, self.on = [], [], 1, 0
        self.devices = []
        cuda = torch.cuda

        @contextlib.contextmanager
        def stream(s):
            was, self.current = self.current, s.cuda_stream
            yield
            self.current = was

        @contextlib.contextmanager
        def device(d):
            was, self.on = self.on, torch.device(d).index
            yield
            self.on = was

        def workspace(n, device="cuda"):
            self.made.append((n, self.current))
            return fake(max(n, 256), dtype=torch.uint8, index=torch.device(device).index or 0)

        def call(name):
            def f(*args):
                self.calls.append((name, args))
                self.devices.append(self.on)
                return workspace_bytes if name.endswith("_size") else W.WISP_OK
            return f

        class Library:
            def __getattr__(self, name):
                return call(name)

        for name, v in (("Stream", FakeStream), ("ExternalStream", lambda raw, device=None: FakeStream(raw)),
                        ("default_stream", lambda device=None: FakeStream(0)), ("stream", stream),
                        ("current_device", lambda: self.on), ("device", device)):
            monkeypatch.setattr(cuda, name, v)
        monkeypatch.setattr(W, "_raw", lambda i: self.current)
        monkeypatch.setattr(W, "workspace", workspace)
        monkeypatch.setattr(W, "lib", Library())
