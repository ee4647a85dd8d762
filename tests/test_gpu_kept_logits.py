"""The 16-bit steps in which the cross entropy's forward keeps logits, measured on the
entries of dL/dz themselves.

The first V columns of W are the identity (times 1) where the hidden states are 0, so that
dhidden_t,v = g_tv, the entries that the two products read; the logits come from four more columns and
are exact in fp32.  All rows have the same logits and weights w_t drawn over a factor of two, so that
the rounding of g to bf16 (2^-8 at most, mean 0) averages out over the rows: the mean over n = 16384 of
them is off by more than 2e-4 with a probability of 2 exp(-n (2e-4)^2 / (2 (2^-8)^2)) = 1e-9 (Hoeffding),
4e-6 for all columns and cases.

What is left of a column's entry against w_t e^(z - lse) is the step's half, 2^-11 in log2, and the
rounding of the row's maximum and of its lse to fp32 and of both times log2 e: 2^-24 each, of at most
1.45 (max + 12), four of them."""
import math

import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("top", [2, 30, 100, 256])
@pytest.mark.parametrize("V", [512, 500])
def test_half_a_step(V, top):
    T, H = 16384, 640
    g = torch.Generator().manual_seed(top + V)
    steps = torch.randint(0, 512, (V,), generator=g)          # z = top - steps / 64
    W = torch.zeros(V, H)
    W[:, :V] = torch.eye(V)
    W[:, 512], W[:, 513], W[:, 514] = 1.0, -(steps // 32) * 0.5, -(steps % 32) / 64.0
    h = torch.zeros(T, H)
    h[:, 512], h[:, 513], h[:, 514] = float(top), 1.0, 1.0
    z = top - steps.double() / 64.0
    assert torch.equal(W, W.to(torch.bfloat16).float()) and torch.equal(h, h.to(torch.bfloat16).float())
    weight = 1.0 + torch.rand(T, generator=g)
    x = torch.randint(0, 8, (T,), generator=g, dtype=torch.int32)
    out = molt.cross_entropy_fwd_bwd(h.to(torch.bfloat16).to(dev()), W.to(torch.bfloat16).to(dev()), x.to(dev()),
                                     token_weight=weight.to(dev()), denom=1.0)
    p = torch.softmax(z, 0).to(dev())
    got = (out["dhidden"][:, :V].double() / weight.to(dev(), torch.float64)[:, None]).mean(0)[8:]   # columns that are nobody's target
    off = (got / p[8:] - 1.0).abs().max()
    bound = 2.0**-11 * math.log(2.0) + 2e-4 + 4 * 2.0**-24 * 1.45 * (top + 12.0)
    assert off <= bound, f"{float(off):.2e}, bound {bound:.2e}"
    assert molt.device_status() == 0
