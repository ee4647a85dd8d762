"""Workspace sizes that the binding keeps: by device, and asked for with that device as the current one."""
import contextlib
import types

import torch

from paper_2607_21653_gb300 import blocks as B


def test_sizes_belong_to_a_device(monkeypatch):
    current, asked = [0], []

    @contextlib.contextmanager
    def device(d):
        current.append(d.index)
        yield
        current.pop()

    def query(ref, *more):
        asked.append((current[-1], more))
        return 1000 * (1 + current[-1])

    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(B, "load", lambda: types.SimpleNamespace(q=query))
    monkeypatch.setattr(B, "_desc_cache", {})
    values = (4, 64, 128, 0, 0, 0, 0, 0, 0, 0)
    for _ in range(2):
        for i in range(2):
            dev = torch.device("cuda", i)
            ref, nbytes = B._desc(dev, B.FfnDesc, values, "q", 1)
            assert nbytes == 1000 * (1 + i) and ref._obj.H == 64
            assert B._desc(dev, B.FfnDesc, values)[1] == 0
    assert asked == [(0, (1,)), (1, (1,))]
