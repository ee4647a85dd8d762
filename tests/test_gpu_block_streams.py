"""`stream` of the operators inside a block: what a call returns is allocated and filled on that stream.

The current stream is held back by a kernel that counts clocks (a tenth of a second), so that what a call
should not have put there comes too late, and memory that is still read there is not to be written."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
HOLD = 200_000_000   # clocks
NAMES = ["ffn", "ffn few", "ffn bwd", "ffn bwd added", "scan", "scan bwd", "step", "dropout", "dropout bwd"]


def calls():
    """Every operator, by name, on inputs of one size."""
    g = torch.Generator(device=dev()).manual_seed(1)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    T, H, F = 512, 512, 1024
    x, dy, gate = n(T, H).to(BF), n(T, H).to(BF), n(T, H).to(BF)
    w, wd = (n(F, H) * H ** -0.5).to(BF), (n(H, F) * F ** -0.5).to(BF)
    states = molt.gated_scan_fwd(gate, x, want_states=True)["states"]
    state = n(T, H)
    return {
        "ffn": lambda **k: molt.gated_ffn_fwd(x, w, w, wd, keep=True, **k),
        "ffn few": lambda **k: molt.gated_ffn_fwd(x[:5], w, w, wd, keep=True, **k),
        "ffn bwd": lambda **k: molt.gated_ffn_bwd(dy, x, w, w, wd, **k),
        "ffn bwd added": lambda **k: molt.gated_ffn_bwd(dy, x, w, w, wd, accumulate=True, **k),
        "scan": lambda **k: molt.gated_scan_fwd(gate, x, want_states=True, **k),
        "scan bwd": lambda **k: molt.gated_scan_bwd(dy, gate, x, states, initial_state=state[:1], **k),
        "step": lambda **k: molt.gated_scan_step(gate, x, state, **k),
        "dropout": lambda **k: {"out": molt.dropout_fwd(x, 0.1, 7, **k)},
        "dropout bwd": lambda **k: {"out": molt.dropout_bwd(dy, 0.1, 7, **k)},
    }


def held(out):
    return {k: t for k, t in out.items() if t is not None}


@pytest.mark.parametrize("name", NAMES)
def test_outputs_belong_to_the_stream(name):
    f = calls()[name]
    want = held(f())
    shapes = [(t.shape, t.dtype) for t in want.values()]
    s = torch.cuda.Stream()
    f(stream=s)                       # (workspaces, and s's own pool)
    torch.cuda.synchronize()
    here = [torch.full(shape, 3.0, device=dev()).to(dtype) for shape, dtype in shapes for _ in range(3)]
    read = [torch.empty_like(t) for t in here]
    torch.cuda.synchronize()
    torch.cuda._sleep(HOLD)
    for i, t in enumerate(here):
        read[i].copy_(t)              # still to come
    del here, t
    out = held(f(stream=s))
    s.synchronize()
    assert not torch.cuda.current_stream().query(), "the current stream was not held back for long enough"
    with torch.cuda.stream(s):
        assert set(out) == set(want)
        for k, v in want.items():
            assert torch.equal(out[k], v), k
    torch.cuda.synchronize()
    assert all((t == 3).all() for t in read)
    for k, v in want.items():
        assert torch.equal(out[k], v), k


def test_captured_on_a_stream_that_is_not_the_current_one():
    """The graph's workspaces are its own, whatever larger calls on the same stream do to the binding's."""
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    fs = calls()
    want = {n: held(f()) for n, f in fs.items()}
    for f in fs.values():
        f(stream=s)
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), {}
    with torch.cuda.graph(graph, stream=s):
        with torch.cuda.stream(other):
            for n, f in fs.items():
                out[n] = held(f(stream=s))
    g = torch.Generator(device=dev()).manual_seed(2)
    x = torch.randn(4096, 1024, device=dev(), generator=g).to(BF)
    w = torch.randn(2048, 1024, device=dev(), generator=g).to(BF)
    for _ in range(2):
        molt.gated_ffn_bwd(x, x, w, w, w.t().contiguous(), stream=s)
        junk = [torch.full((1 << 22,), 9.0, device=dev()) for _ in range(8)]
        for t in (t for o in out.values() for t in o.values()):
            t.zero_()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph.replay()
        torch.cuda.synchronize()
        for n, o in want.items():
            for k, v in o.items():
                assert torch.equal(out[n][k], v), (n, k)
        assert all((t == 9).all() for t in junk)
    assert molt.device_status() == 0
