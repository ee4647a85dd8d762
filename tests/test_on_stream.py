"""`stream` of the calls: their whole body runs with it as the current stream."""
import contextlib
import inspect

import pytest
import torch

import paper_2607_21653_gb300 as molt

NAMES = ["gated_ffn_fwd", "gated_ffn_bwd", "gated_scan_fwd", "gated_scan_bwd", "gated_scan_step", "dropout_fwd", "dropout_bwd"]


@pytest.fixture
def current(monkeypatch):
    """torch.cuda.stream without a device: the stack of streams."""
    stack = []

    @contextlib.contextmanager
    def stream(s):
        stack.append(s)
        yield
        stack.pop()

    monkeypatch.setattr(torch.cuda, "stream", stream)
    return stack


def test_the_body_runs_on_the_stream(current):
    seen = []

    @molt._on_stream
    def f(x, y=1, stream=None, workspace=None):
        seen.append((x, y, stream, workspace, list(current)))
        return x

    assert [f(1), f(2, 3, "s"), f(4, stream="t", workspace=5), f(6, stream=None)] == [1, 2, 4, 6]
    assert seen == [(1, 1, None, None, []), (2, 3, "s", None, ["s"]), (4, 1, "t", 5, ["t"]), (6, 1, None, None, [])]
    assert list(inspect.signature(f).parameters) == ["x", "y", "stream", "workspace"]
    with pytest.raises(TypeError):
        f()


@pytest.mark.parametrize("name", NAMES)
def test_refusals_come_from_inside_it(current, name):
    """(tensors on the host are refused, with the stream as the current one)"""
    f = getattr(molt, name)
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w, wd = torch.zeros(128, 64, dtype=torch.bfloat16), torch.zeros(64, 128, dtype=torch.bfloat16)
    args = {"gated_ffn_fwd": (x, w, w, wd), "gated_ffn_bwd": (x, x, w, w, wd), "gated_scan_fwd": (x, x), "gated_scan_bwd": (x, x, x, x),
            "gated_scan_step": (x, x, x.float()), "dropout_fwd": (x, 0.1, 1), "dropout_bwd": (x, 0.1, 1)}[name]
    entered = []
    real = torch.cuda.stream

    def stream(s):
        entered.append(s)
        return real(s)

    torch.cuda.stream = stream
    try:
        with pytest.raises(TypeError, match="CUDA"):
            f(*args, stream="s")
    finally:
        torch.cuda.stream = real
    assert entered == ["s"]


def test_every_call_with_a_stream():
    for name in molt.__all__:
        f = getattr(molt, name)
        if callable(f) and not inspect.isclass(f) and "stream" in inspect.signature(f).parameters:
            assert hasattr(f, "__wrapped__") != (name in ("device_status", "selftest_wait_timeout")), name
