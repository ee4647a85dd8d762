"""The feed-forward block's gradients where gate products are large: act' is 0 or 1 there, act(g) 0 or g, whatever
their powers are.

Tolerances: one row in and one weight a time (H = F = 8, diagonal weights of 1), so every sum has one term; a result is
a chain of at most three roundings to bf16 (dh, dg or du or h, and the result), 3 (2^-8) of it, and act and
act' are off by 2^-17.  Sizes stay below bf16's largest."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
GATES = [1e4, 3e9, 1e20, 1e30, 1e38, 30.0, 6.0, 0.0]


def act64(name, g):
    if name == "relu":
        return g.clamp(min=0), (g > 0).double()
    z = g.clamp(-60, 60)   # (act' is 0 or 1 to all digits from there on, and act(g) = act'(g) g)
    z = z.detach().requires_grad_(True)
    a = torch.nn.functional.silu(z) if name == "silu" else torch.nn.functional.gelu(z, approximate="tanh")
    d, = torch.autograd.grad(a.sum(), z)
    return torch.where(g.abs() > 60, (g > 0) * g, a.detach()), torch.where(g.abs() > 60, (g > 0).double(), d)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("rows", [1, 40])
def test_gradients_of_large_gates(act, sign, rows):
    n = 8
    eye = torch.eye(n, dtype=BF, device=dev())
    g = (sign * torch.tensor(GATES, device=dev())).to(BF).expand(rows, n).contiguous()
    small = torch.full((rows, n), 2.0**-10, dtype=BF, device=dev())
    x = torch.full((rows, n), 0.5, dtype=BF, device=dev())
    a, d = act64(act, g.double())
    # kept products: the gates as they are
    out = molt.gated_ffn_bwd(small, x, eye, eye, eye, g, small, activation=act, dw_dtype=torch.float32)
    dg, du, h = 2.0**-20 * d, 2.0**-10 * a, a * 2.0**-10
    tol = 3 * 2.0**-8 + 2.0**-16
    near = lambda got, want, extra=0.0: bool(((got.double() - want).abs() <= tol * want.abs() + extra).all())
    assert near(out["dx"], dg + du, tol * dg.abs().max()), act
    want = rows * 0.5
    assert near(torch.diagonal(out["dw_gate"]), want * dg[0], 1e-30) and near(torch.diagonal(out["dw_up"]), want * du[0], 1e-30)
    assert near(torch.diagonal(out["dw_down"]), rows * 2.0**-10 * h[0], 1e-30)
    # formed by the call: the gates are x itself, u = 2^-126 of them (h = 1e76 2^-126 = 1.2e38 at most: past
    # bf16's largest, 3.4e38, h would be infinite and the product with zeros NaN)
    fwd = molt.gated_ffn_fwd(g, eye, (eye.float() * 2.0**-126).to(BF), eye, activation=act)
    assert near(fwd["y"], a * (g.double() * 2.0**-126), 1e-37)
