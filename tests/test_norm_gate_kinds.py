"""What a gate's shape says where there are as many rows as channels."""
import importlib.util
import os

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300 import stream as S

BF, F = torch.bfloat16, torch.float32


def test_a_vector_that_could_be_either_is_refused():
    x, w = torch.zeros(64, 64, dtype=BF), torch.ones(64)
    for gate in (torch.ones(64), torch.ones(64, 64)[0]):
        with pytest.raises(ValueError, match="gate_kind"):
            molt.residual_norm_fwd(x, gate=gate, w_pre=w)
        with pytest.raises(ValueError, match="gate_kind"):
            molt.residual_norm_bwd(x, None, x, x, w, gate=gate, w_pre=w)
    # past the gate: the tensors are on the host
    for kw in (dict(gate=w, gate_kind="channel"), dict(gate=w, gate_kind="token"), dict(gate=w[:, None]),
               dict(gate=torch.ones(64, dtype=BF), w_pre=torch.ones(64, dtype=BF)), dict(gate=torch.ones(64, 64, dtype=BF))):
        with pytest.raises(TypeError, match="CUDA"):
            molt.residual_norm_fwd(x, **{"w_pre": w, **kw})


@pytest.mark.parametrize("T,H,shape,dtype,want", [
    (4, 64, (64,), F, S.GATE_CHANNEL), (4, 64, (4,), F, S.GATE_TOKEN), (4, 64, (4, 1), F, S.GATE_TOKEN), (4, 64, (4, 64), BF, S.GATE_FULL),
    (64, 64, (64, 1), F, S.GATE_TOKEN), (64, 64, (64,), BF, S.GATE_CHANNEL), (64, 64, (64, 64), F, S.GATE_FULL),
    (1, 1, (1,), F, S.GATE_CHANNEL), (1, 64, (1, 64), BF, S.GATE_FULL), (0, 64, (64,), F, S.GATE_CHANNEL)])
def test_kind_by_shape(T, H, shape, dtype, want):
    assert S._gate_kind(torch.ones(shape, dtype=dtype), T, H) == want


def test_a_stated_kind_has_to_fit():
    g = torch.ones(64)
    assert S._gate_kind(g, 64, 64, "token") == S.GATE_TOKEN and S._gate_kind(g, 64, 64, "channel") == S.GATE_CHANNEL
    assert S._gate_kind(torch.ones(64, 1, dtype=BF), 64, 1, "full") == S.GATE_FULL
    for shape, kind in (((64,), "token"), ((4,), "channel"), ((4, 1), "full"), ((64,), "row")):
        with pytest.raises(ValueError, match="gate"):
            S._gate_kind(torch.ones(shape), 4, 64, kind)
    with pytest.raises(ValueError, match="gate"):
        S._gate_kind(None, 4, 64, "token")


@pytest.mark.gpu
def test_as_many_rows_as_channels():
    """The same gate as [T, 1] and, with its kind stated, as [T]; and as a channel's."""
    T = H = 320
    g = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x, r, w, gate, dy = n(T, H).to(BF), n(T, H), 1 + 0.1 * n(H), n(T), n(T, H).to(BF)

    def both(gate, **kw):
        o = molt.residual_norm_fwd(x, r, gate=gate, w_pre=w, **kw)
        b = molt.residual_norm_bwd(dy, None, x, o["residual"], o["rstd_pre"], gate=gate, w_pre=w, **kw)
        return {**o, **b}

    token, stated, channel = both(gate[:, None]), both(gate, gate_kind="token"), both(gate, gate_kind="channel")
    for k, v in token.items():
        assert v is None or torch.equal(v, stated[k]), k
    # r' is one fused multiply-add, rounded once: 2^-24 of its terms' sum and of u's own rounding
    for out, g2 in ((token, gate[:, None]), (channel, gate[None, :])):
        want = r.double() + g2.double() * x.double()
        assert ((out["residual"].double() - want).abs() <= 2.0**-22 * (r.double().abs() + (g2 * x).double().abs())).all()


@pytest.mark.gpu
def test_example_with_as_many_tokens_as_channels():
    """Its gate vectors are fp32 and a channel's for every number of tokens."""
    spec = importlib.util.spec_from_file_location(
        "warm_start", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "warm_start.py"))
    warm_start = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(warm_start)
    policy = warm_start.Policy(512, 128, 1)
    tokens, targets = warm_start.batch(128, 512, torch.Generator(device="cuda").manual_seed(1))
    loss, grads = policy.step(tokens, targets)
    assert torch.isfinite(loss).all() and grads["gate0"].shape == (128,)
