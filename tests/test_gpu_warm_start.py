"""The supervised step of examples/warm_start.py: its gradients against autograd in fp64,
and the fit itself.

Tolerance, before any run: the step rounds to bf16 (2^-9 of a value, 2e-3 in the mean) the
embedding, each block's four products and norms and, on the way back, as many gradients:
some 12 independent roundings at one block, 24 at two, so about 1 % of a gradient in the
mean, 5 times that for the largest error of many entries: 5e-2 of the largest entry, a
cosine of at least 0.999.  Where rounding turns the sign of a relu's input the gradient
jumps, so the reference takes the step's own branches."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location(
    "warm_start", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "warm_start.py"))
warm_start = importlib.util.module_from_spec(spec)
spec.loader.exec_module(warm_start)


def reference(policy, tokens, targets, e, c):
    p = {k: v.double().clone().requires_grad_(True) for k, v in policy.w.items()}
    rms = lambda z, w: z * torch.rsqrt((z * z).mean(1, keepdim=True) + 1e-6) * w
    open_ = [h > 0 for _, _, h, _ in policy.forward(tokens)[1][1:]]
    r = p["W"][tokens.long()] * policy.scale
    y = rms(r, p["norm0"])
    for i in range(policy.blocks):
        o = ((y @ p[f"A{i}"]) * open_[i]) @ p[f"B{i}"]
        r = r + p[f"gate{i}"] * rms(o, p[f"post{i}"])
        y = rms(r, p[f"norm{i + 1}"])
    z = y @ p["W"].t()
    act = targets != -100
    lse = torch.logsumexp(z, 1)
    zx = z.gather(1, targets.long().clamp(min=0)[:, None])[:, 0]
    loss = ((lse - (1 - e) * zx - e * z.mean(1) + c * lse * lse) * act).sum() / act.sum()
    loss.backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("T,H,V,blocks,e,c", [(1, 64, 64, 1, 0.0, 0.0), (300, 128, 512, 1, 0.0, 0.0), (301, 192, 1000, 2, 0.1, 1e-3),
                                            (700, 640, 900, 2, 0.0, 0.0)])
def test_gradients(T, H, V, blocks, e, c):
    policy = warm_start.Policy(V, H, blocks, device=dev(), seed=T)
    gen = torch.Generator(device=dev()).manual_seed(T)
    tokens, targets = warm_start.batch(T, V, gen, device=dev())
    if T == 1:
        targets[:] = 5
    loss, grads = policy.step(tokens, targets, label_smoothing=e, z_loss=c)
    ref_loss, ref = reference(policy, tokens, targets, float(np.float32(e)), float(np.float32(c)))
    assert set(grads) == set(ref)
    assert abs(float(loss) - float(ref_loss)) <= 1e-2 * float(ref_loss)
    for k, g in grads.items():
        g, r = g.double().flatten(), ref[k].flatten()
        assert (g - r).abs().max() <= 5e-2 * r.abs().max(), k
        assert float((g * r).sum() / (g.norm() * r.norm())) >= 0.999, k
    assert molt.device_status() == 0


def test_fits(capsys):
    losses, held_out = warm_start.main(["--steps", "40", "--tokens", "1024", "--hidden", "256", "--vocab", "2048"])
    assert losses[0] > 0.5 * math.log(2048)
    assert held_out < 0.25 * losses[0]
    line = capsys.readouterr().out.strip().splitlines()[-1].split()
    assert abs(float(line[3]) - float(line[6])) <= 2e-3   # the two forwards' log-probabilities
