"""Supervised warm start of a small policy with tied embeddings, on the library's calls.

Before the policy update of a run has rollouts to learn from, the policy is fitted to
demonstrations by the cross entropy of their next tokens.  One step here is

    x    = embedding of the tokens                                token_embedding
    r, y = residual stream (fp32), its norm                       residual_norm_fwd
    per block: o = relu(y A) B                                    torch
               r = r + gate * norm(o),  y = norm(r)               residual_norm_fwd
    loss, its gradient to y and the head's dW                     cross_entropy_fwd_bwd
    the blocks backwards                                          residual_norm_bwd
    the embedding's gradient, added to the same dW                token_embedding_bwd

and an SGD update with momentum.  The head's weights are the embedding (tied), so the last two
gradients land in one fp32 dW.  After the fit the log-probabilities that the policy
update's forward gives for the same tokens are compared with the loss.

    python examples/warm_start.py [--steps 60] [--tokens 4096] [--hidden 512] [--vocab 8192] [--blocks 2]

The data are synthetic: a target follows its token by a fixed permutation, one token in
ten is not a target (ignored).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2607_21653_gb300 as molt  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


class Policy:
    """fp32 parameters, and bf16 copies of the matrices that the steps use."""

    def __init__(self, V, H, blocks, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        normal = lambda *s, std: torch.randn(*s, device=device, generator=g) * std
        self.V, self.H, self.blocks = V, H, blocks
        self.p = {"W": normal(V, H, std=H ** -0.5), "norm0": torch.ones(H, device=device)}
        for i in range(blocks):
            self.p[f"A{i}"] = normal(H, 2 * H, std=H ** -0.5)
            self.p[f"B{i}"] = normal(2 * H, H, std=(2 * H) ** -0.5)
            self.p[f"post{i}"] = torch.ones(H, device=device)
            self.p[f"gate{i}"] = torch.full((H,), 0.5, device=device)
            self.p[f"norm{i + 1}"] = torch.ones(H, device=device)
        self.scale = H ** 0.5
        self.cast()

    def cast(self):
        self.w = {k: v.to(BF16) if v.dim() == 2 else v for k, v in self.p.items()}

    def forward(self, tokens):
        """The hidden states for the head, and what the backward needs."""
        w, kept = self.w, []
        x = molt.token_embedding(w["W"], tokens, scale=self.scale)
        s = molt.residual_norm_fwd(x, w_pre=w["norm0"], residual_dtype=F32)
        kept.append((x, None, None, s))
        for i in range(self.blocks):
            y = s["y"]
            h = torch.relu(y @ w[f"A{i}"])
            o = h @ w[f"B{i}"]
            s = molt.residual_norm_fwd(o, s["residual"], w_post=w[f"post{i}"], gate=w[f"gate{i}"], w_pre=w[f"norm{i + 1}"],
                                       gate_kind="channel")
            kept.append((o, y, h, s))
        return s["y"], kept

    def step(self, tokens, targets, label_smoothing=0.0, z_loss=0.0):
        """Loss and the gradients of all parameters (fp32; the blocks' matrices bf16)."""
        w, grads = self.w, {}
        y, kept = self.forward(tokens)
        out = molt.cross_entropy_fwd_bwd(y, w["W"], targets, label_smoothing=label_smoothing, z_loss=z_loss)
        dy, dr = out["dhidden"], None
        for i in reversed(range(self.blocks)):
            o, y, h, s = kept[i + 1]
            b = molt.residual_norm_bwd(dy, dr, o, s["residual"], s["rstd_pre"], s["rstd_post"], w_post=w[f"post{i}"],
                                       gate=w[f"gate{i}"], w_pre=w[f"norm{i + 1}"], gate_kind="channel")
            do, dr = b["dx"], b["dresidual"]
            grads[f"post{i}"], grads[f"gate{i}"], grads[f"norm{i + 1}"] = b["dw_post"], b["dgate"], b["dw_pre"]
            grads[f"B{i}"] = h.t() @ do
            dh = (do @ w[f"B{i}"].t()) * (h > 0)
            grads[f"A{i}"] = y.t() @ dh
            dy = dh @ w[f"A{i}"].t()
        x, _, _, s = kept[0]
        b = molt.residual_norm_bwd(dy, dr, x, s["residual"], s["rstd_pre"], w_pre=w["norm0"], want_dresidual=False)
        grads["norm0"] = b["dw_pre"]
        # the head's dW and the embedding's, in one buffer
        grads["W"] = molt.token_embedding_bwd(b["dx"], tokens, self.V, scale=self.scale, dW=out["dW"], accumulate_dW=True)
        return out["loss"], grads

    def update(self, grads, state, lr, momentum=0.9, clip=1.0):
        norm = torch.sqrt(sum((g.float() ** 2).sum() for g in grads.values()))
        f = torch.clamp(clip / norm, max=1.0)
        for k, g in grads.items():
            m = state.setdefault(k, torch.zeros_like(self.p[k]))
            m.mul_(momentum).add_(g.float() * f)
            self.p[k].sub_(lr * m)
        self.cast()


def batch(T, V, gen, device="cuda"):
    """Tokens of 64 frequent ids and their targets."""
    tokens = torch.randint(0, 64, (T,), device=device, generator=gen) * (V // 64)
    targets = (tokens * 5 + 3) % V
    targets[torch.rand(T, device=device, generator=gen) < 0.1] = -100
    return tokens.to(torch.int32), targets.to(torch.int32)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    for name, value in (("steps", 60), ("tokens", 4096), ("hidden", 512), ("vocab", 8192), ("blocks", 2)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    if a.vocab < 64 or a.hidden % 64:
        ap.error("--vocab is at least 64, --hidden a multiple of 64")
    policy, state = Policy(a.vocab, a.hidden, a.blocks), {}
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for i in range(a.steps):
        tokens, targets = batch(a.tokens, a.vocab, gen)
        loss, grads = policy.step(tokens, targets)
        policy.update(grads, state, a.lr)
        losses.append(float(loss))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {losses[-1]:.4f}")
    # the same hidden states in the policy update's forward
    tokens, targets = batch(a.tokens, a.vocab, gen)
    y, _ = policy.forward(tokens)
    out = molt.cross_entropy_fwd(y, policy.w["W"], targets)
    mask = (targets != -100).to(torch.uint8)
    logp, _ = molt.token_logprobs(y, policy.w["W"], targets, mask)
    print(f"held out  loss {float(out['loss']):.4f}  from token_logprobs {-float(logp.double().sum() / mask.sum()):.4f}")
    return losses, float(out["loss"])


if __name__ == "__main__":
    main()
