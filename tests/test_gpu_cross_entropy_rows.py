"""Cross entropy's gradient row by row, each measured against the row's own size: rows that
the model predicts well, whose losses run from 1 to 1e-5, have gradients as small as their
losses, which a bound against the largest entry of the matrix does not see.

Bounds, before any run.  With w / D = 1 a row's dhidden is sum_v g_v W_v, g_v = p_v - [v = x],
and its error in the 2-norm is at most the sum of
  * g rounded to bf16 (2^-8), taken from kept logits (2^-11 ln 2) and from fp32 logits and
    row sums that are good to a few 1e-5 at the most (2^-12):  each times sum_v |g_v| |W_v|;
  * the target's p - 1, which is 1 less the rest of fp32 sums of numbers up to 1 and of
    approximate exponentials (2^-22 each): 2^-20 |W_x|;
  * the result's own rounding to bf16: 2^-8 of it.
logp is good to that 2^-20 and to the logits' own 2^-15 where p is not near 1."""
import math

import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu
SHAPES = [(64, 500), (512, 3000), (1024, 20000), (4096, 5003)]


def predicted_rows(T, H, V, seed):
    """Rows whose target is ahead of all others together by 0 to 12."""
    g = torch.Generator().manual_seed(seed)
    W = (torch.randn(V, H, generator=g) * 0.02).to(torch.bfloat16)
    x = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    Wx = W[x.long()].double()
    others = math.log(V) + 0.5 * 4e-4 * H
    boost = (others + 12.0 * torch.arange(T) / T) / Wx.square().sum(1)
    h = torch.randn(T, H, generator=g).double() + boost[:, None] * Wx
    return h.to(torch.bfloat16).to(dev()), W.to(dev()), x.to(dev())


def reference(h, W, x, e, c):
    """(g, logp, dhidden, dW) in fp64, the target's entry of g from the others' sum."""
    h, W, x = h.double(), W.double(), x.long()[:, None]
    z = h @ W.t()
    lse = torch.logsumexp(z, 1, keepdim=True)
    rest = z.scatter(1, x, float("-inf"))
    p = torch.exp(rest - lse)
    left = p.sum(1, keepdim=True)                       # 1 - p_x, without a difference
    cp = 1.0 + 2.0 * c * lse
    g = p * cp - e / W.shape[0]
    g.scatter_(1, x, -left + 2.0 * c * lse * (1.0 - left) + e - e / W.shape[0])
    return g, torch.log1p(-left)[:, 0], left[:, 0], g @ W, g.t() @ h


@pytest.mark.parametrize("H,V", SHAPES)
def test_log_probs_of_predicted_rows(H, V):
    h, W, x = predicted_rows(700, H, V, seed=H + V)
    _, logp, left, _, _ = reference(h, W, x, 0.0, 0.0)
    assert left.min() < 5e-5 and left.max() > 0.3   # what the rows are meant to be
    far = (molt.cross_entropy_fwd(h, W, x)["logp"].double() - logp).abs()
    lim = 2.0**-20 + 2.0**-15 * left
    assert (far <= lim).all(), f"logp: {float((far / lim).max()):.2f} of the bound"


@pytest.mark.parametrize("H,V", SHAPES)
@pytest.mark.parametrize("e,c", [(0.0, 0.0), (0.0, 2.0**-20), (2.0**-14, 0.0)])
def test_gradient_of_predicted_rows(H, V, e, c):
    T = 700
    h, W, x = predicted_rows(T, H, V, seed=H + V)
    g, _, left, dh, dW = reference(h, W, x, e, c)
    out = molt.cross_entropy_fwd_bwd(h, W, x, denom=1.0, label_smoothing=e, z_loss=c)
    size = W.double().norm(dim=1)
    entry = 2.0**-8 + 2.0**-11 * math.log(2.0) + 2.0**-12
    lim = entry * (g.abs() @ size) + 2.0**-20 * size[x.long()] + 2.0**-8 * dh.norm(dim=1)
    far = (out["dhidden"].double() - dh).norm(dim=1)
    assert (far <= lim).all(), f"dhidden: {float((far / lim).max()):.2f} of the bound at a row whose p is {1 - float(left[(far / lim).argmax()]):.7f}"
    # column sums of the same entries
    hs = h.double().norm(dim=1)
    onehot = torch.zeros(V, T, dtype=torch.float64, device=dev()).scatter_(0, x.long()[None, :], 1.0)
    lim = entry * (g.abs().t() @ hs) + 2.0**-20 * (onehot @ hs) + 2.0**-16 * (g.abs().t() @ hs)
    far = (out["dW"].double() - dW).norm(dim=1)
    assert (far <= lim).all(), f"dW: {float((far / lim).max()):.2f} of the bound"
    assert molt.device_status() == 0


@pytest.mark.parametrize("ahead", [20.0, 200.0, 20000.0])
def test_a_target_far_ahead_of_the_others(ahead):
    """Nothing is left of the others: no loss, and no gradient beyond the bound's 2^-20."""
    T, H, V = 40, 640, 700
    g = torch.Generator().manual_seed(3)
    W = (torch.randn(V, H, generator=g) * 0.02).to(torch.bfloat16)
    x = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    h = (W[x.long()].float() * (ahead / (H * 4e-4) * 2.0)).to(torch.bfloat16).to(dev())
    W, x = W.to(dev()), x.to(dev())
    z = h.double() @ W.double().t()
    left = torch.exp(z - torch.logsumexp(z, 1, keepdim=True)).scatter(1, x.long()[:, None], 0.0).sum(1)
    out = molt.cross_entropy_fwd_bwd(h, W, x, denom=1.0)
    assert torch.isfinite(out["logp"]).all() and (out["logp"].double().abs() <= 2.0**-20 + 2.0 * left).all()
    zx = z.gather(1, x.long()[:, None])[:, 0]
    assert ((out["lse"].double() - zx).abs() <= 2.0**-20 + 2.0 * left + 2.0**-18 * zx).all()
    size = W.double().norm(dim=1)
    lim = (2.0**-20 + 4.0 * left) * (size[x.long()] + size.max()) * 1.01
    assert (out["dhidden"].double().norm(dim=1) <= lim).all()
