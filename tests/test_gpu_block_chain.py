"""The operators inside a block together: the gated blocks of examples/warm_start.py against
autograd in fp64 and against its decode token by token, and a block forward and backward in captured
graphs.

Tolerance of the gradients, before any run: a block rounds to bf16 (2^-9 of a value, 2e-3 in the
mean of a vector) its projection, the recurrence, two dropped copies, two norms, h, the kept
products and the block's output, some 9, and as many gradients on the way back: 18 a block,
36 at two, so 2e-3 sqrt(36) = 1.2 % of a gradient in the mean and, of many entries,
4 times that for the largest: 5e-2 of the largest entry, a cosine of at least 0.999.

Of the decode: it rounds where the forward does, and where sums are taken in another order a
rounding may fall the other way: a few of 9 roundings a block, each 2e-3 in the mean, against a
stream that carries the embedding besides: 1e-2 normwise."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

spec = importlib.util.spec_from_file_location(
    "warm_start", os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples", "warm_start.py"))
warm_start = importlib.util.module_from_spec(spec)
spec.loader.exec_module(warm_start)


def cuts(T, lengths):
    return torch.tensor([0, *np.minimum(np.cumsum(lengths), T)], dtype=torch.int32, device=dev())


def reference(policy, tokens, targets):
    p = {k: v.double().clone().requires_grad_(True) for k, v in policy.w.items()}
    H, T = policy.H, tokens.numel()
    rms = lambda z, w: z * torch.rsqrt((z * z).mean(1, keepdim=True) + 1e-6) * w
    first = set(policy.cu_seqlens.tolist())
    kept = lambda m: molt.dropout_fwd(torch.ones(T, H, device=dev()), **m).double()
    r = p["W"][tokens.long()] * policy.scale
    y = rms(r, p["norm0"])
    for i in range(policy.blocks):
        m1, m2 = policy.masks(i)
        fv = y @ p[f"G{i}"]
        a, rows = torch.sigmoid(fv[:, :H]), []
        for t in range(T):
            b = (1 - a[t]) * fv[t, H:]
            rows.append(b if t in first else a[t] * rows[-1] + b)
        r = r + torch.stack(rows) * kept(m1)
        y = rms(r, p[f"mid{i}"])
        f = torch.nn.functional.silu(y @ p[f"Wg{i}"].t()) * (y @ p[f"Wu{i}"].t())
        r = r + (f @ p[f"Wd{i}"].t()) * kept(m2)
        y = rms(r, p[f"norm{i + 1}"])
    z = y @ p["W"].t()
    act = targets != -100
    loss = ((torch.logsumexp(z, 1) - z.gather(1, targets.long().clamp(min=0)[:, None])[:, 0]) * act).sum() / act.sum()
    loss.backward()
    return loss.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("T,H,V,blocks,p,lengths", [(1, 64, 64, 1, 0.1, [1]), (300, 128, 512, 1, 0.1, [1, 129, 0, 170]),
                                                    (301, 192, 1000, 2, 0.25, [128, 128, 45]), (700, 640, 900, 2, 0.0, [700])])
def test_gradients(T, H, V, blocks, p, lengths):
    policy = warm_start.GatedPolicy(V, H, blocks, device=dev(), seed=T, p=p)
    policy.cu_seqlens, policy.draw = cuts(T, lengths), 3
    gen = torch.Generator(device=dev()).manual_seed(T)
    tokens, targets = warm_start.batch(T, V, gen, device=dev())
    if T == 1:
        targets[:] = 5
    loss, grads = policy.step(tokens, targets)
    ref_loss, ref = reference(policy, tokens, targets)
    assert set(grads) == set(ref)
    assert abs(float(loss) - float(ref_loss)) <= 1e-2 * float(ref_loss)
    for k, g in grads.items():
        g, r = g.double().flatten(), ref[k].flatten()
        assert (g - r).abs().max() <= 5e-2 * r.abs().max(), k
        assert float((g * r).sum() / (g.norm() * r.norm()).clamp(min=1e-300)) >= (0.999 if float(r.norm()) > 0 else 0), k
    assert molt.device_status() == 0


def test_decode_continues_the_forward():
    """Three sequences decoded side by side from the states that the forward left."""
    H, V, L, more = 256, 512, 130, 6
    policy = warm_start.GatedPolicy(V, H, 2, device=dev(), seed=1, p=0.0)
    gen = torch.Generator(device=dev()).manual_seed(1)
    tokens = torch.randint(0, V, (3, L + more), device=dev(), generator=gen).to(torch.int32)
    policy.cu_seqlens = cuts(3 * (L + more), [L + more] * 3)
    whole = policy.forward(tokens.reshape(-1))[0].view(3, L + more, H)
    states = [torch.zeros(3, H, device=dev()) for _ in range(2)]
    for t in range(L + more):
        y = policy.decode(tokens[:, t].contiguous(), states)
        if t in (0, 1, L, L + more - 1):
            want = whole[:, t].double()
            assert float((y.double() - want).norm() / want.norm()) <= 1e-2, t
    assert molt.device_status() == 0


def test_example_runs(capsys):
    losses, _ = warm_start.main(["--block", "gated", "--steps", "2", "--tokens", "300", "--hidden", "128", "--vocab", "512",
                                 "--length", "128"])
    assert len(losses) == 2 and all(np.isfinite(losses))
    assert "128 tokens decoded" in capsys.readouterr().out


def block(d, seeds, H):
    """A block forward and backward on the binding's own workspaces, everything that comes out."""
    out = {}
    h = molt.gated_scan_fwd(d["fv"][:, :H], d["fv"][:, H:], initial_state=d["h0"], cu_seqlens=d["cu"], want_states=True)
    r1 = molt.dropout_fwd(h["y"], 0.1, seeds[0], residual=d["r"], res_scale=0.5)
    s = molt.residual_norm_fwd(r1, w_pre=d["w"], residual_dtype=F32)
    y = s["y"].to(BF)
    f = molt.gated_ffn_fwd(y, d["wg"], d["wu"], d["wd"], keep=True)
    r2 = molt.dropout_fwd(f["y"], 0.1, seeds[1], residual=r1)
    b = molt.dropout_bwd(d["dr"], 0.1, seeds[1], dtype=BF)
    g = molt.gated_ffn_bwd(b, y, d["wg"], d["wu"], d["wd"], f["gate"], f["up"])
    n = molt.residual_norm_bwd(g["dx"].to(s["y"].dtype), d["dr"], r1, s["residual"], s["rstd_pre"], w_pre=d["w"])
    dh = molt.dropout_bwd(n["dx"], 0.1, seeds[0], dtype=BF)
    z = molt.gated_scan_bwd(dh, d["fv"][:, :H], d["fv"][:, H:], h["states"], initial_state=d["h0"], cu_seqlens=d["cu"])
    for k, v in (("h", h), ("f", f), ("g", g), ("n", n), ("z", z)):
        out.update({k + "_" + name: t for name, t in v.items() if t is not None})
    return {**out, "r1": r1, "r2": r2}


def draw(T, H, F, seed):
    g = torch.Generator(device=dev()).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    cu = torch.cat((torch.zeros(1, device=dev()), torch.rand(2, device=dev(), generator=g).sort().values * T,
                    torch.full((1,), T, device=dev()))).to(torch.int32)
    return dict(fv=n(T, 2 * H).to(BF), h0=n(3, H), cu=cu, r=n(T, H), dr=n(T, H), w=1 + 0.1 * n(H), wg=(n(F, H) * H ** -0.5).to(BF),
                wu=(n(F, H) * H ** -0.5).to(BF), wd=(n(H, F) * F ** -0.5).to(BF))


def test_two_captured_graphs():
    """Graphs of two sizes captured in turn and replayed in either order, on new inputs and with new
    masks, beside calls outside of them that use (and regrow) the stream's own workspaces."""
    sizes = {"a": (700, 256, 704), "b": (20, 512, 1024)}
    held = {k: draw(*v, 1) for k, v in sizes.items()}
    seeds = {k: [torch.tensor([5, i], device=dev()) for i in range(2)] for k in sizes}
    graphs, outs = {}, {}
    for k, (T, H, F) in sizes.items():
        block(held[k], seeds[k], H)
        torch.cuda.synchronize()
        graphs[k] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[k]):
            outs[k] = block(held[k], seeds[k], H)
    masks = []
    for turn, order in enumerate(("ab", "ba", "aab")):
        for k in sizes:
            for name, t in draw(*sizes[k], 10 + turn).items():
                held[k][name].copy_(t)
            for i, t in enumerate(seeds[k]):
                t.copy_(torch.tensor([100 + turn, 7 * i]))
        block(draw(3000, 256, 704, turn), seeds["a"], 256)   # workspaces larger than the graphs' own
        for k in order:
            graphs[k].replay()
        torch.cuda.synchronize()
        for k in sizes:
            got = {n: t.clone() for n, t in outs[k].items()}
            want = block(held[k], seeds[k], sizes[k][1])
            assert set(got) == set(want)
            for n, t in want.items():
                assert torch.equal(t, got[n]), (turn, k, n)
        masks.append(molt.dropout_fwd(torch.ones(64, 64, device=dev()), 0.1, seeds["a"][0]))
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])
    assert molt.device_status() == 0


def test_two_streams_at_once():
    """The block on two streams at the same time, each with workspaces of its own."""
    T, H, F = 1500, 512, 1408
    d = [draw(T, H, F, 20 + i) for i in range(2)]
    want = [block(x, (3, 4), H) for x in d]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in d]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = block(d[i], (3, 4), H)
    torch.cuda.synchronize()
    for i in range(2):
        for n, t in want[i].items():
            assert torch.equal(t, got[i][n]), (i, n)
    assert molt.device_status() == 0
