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
gradients land in one fp32 dW.  With --block gated a block is instead

    f, v = halves of y G                                          torch
    r, y = r + dropout(recurrence(f, v)), its norm                gated_scan_fwd, dropout_fwd, residual_norm_fwd
    r, y = r + dropout((silu(y Wg^T) * y Wu^T) Wd^T), its norm    gated_ffn_fwd, dropout_fwd, residual_norm_fwd

on sequences of --length tokens, and the fit is followed by a decode of one of them token by token
(gated_scan_step), whose hidden states are compared with the forward's.  After the fit the log-probabilities that the policy
update's forward gives for the same tokens are compared with the loss.

    python examples/warm_start.py [--steps 60] [--tokens 4096] [--hidden 512] [--vocab 8192] [--blocks 2]
                                  [--block relu | gated] [--length 512] [--dropout 0.1]

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
            self.make_block(i, H, normal, device)
        self.scale = H ** 0.5
        self.cast()

    def make_block(self, i, H, normal, device):
        self.p[f"A{i}"] = normal(H, 2 * H, std=H ** -0.5)
        self.p[f"B{i}"] = normal(2 * H, H, std=(2 * H) ** -0.5)
        self.p[f"post{i}"] = torch.ones(H, device=device)
        self.p[f"gate{i}"] = torch.full((H,), 0.5, device=device)
        self.p[f"norm{i + 1}"] = torch.ones(H, device=device)

    def cast(self):
        self.w = {k: v.to(BF16) if v.dim() == 2 else v for k, v in self.p.items()}

    def block_fwd(self, i, s):
        w, y = self.w, s["y"]
        h = torch.relu(y @ w[f"A{i}"])
        o = h @ w[f"B{i}"]
        s = molt.residual_norm_fwd(o, s["residual"], w_post=w[f"post{i}"], gate=w[f"gate{i}"], w_pre=w[f"norm{i + 1}"],
                                   gate_kind="channel")
        return s, (o, y, h, s)

    def block_bwd(self, i, kept, dy, dr, grads):
        w, (o, y, h, s) = self.w, kept
        b = molt.residual_norm_bwd(dy, dr, o, s["residual"], s["rstd_pre"], s["rstd_post"], w_post=w[f"post{i}"],
                                   gate=w[f"gate{i}"], w_pre=w[f"norm{i + 1}"], gate_kind="channel")
        do, dr = b["dx"], b["dresidual"]
        grads[f"post{i}"], grads[f"gate{i}"], grads[f"norm{i + 1}"] = b["dw_post"], b["dgate"], b["dw_pre"]
        grads[f"B{i}"] = h.t() @ do
        dh = (do @ w[f"B{i}"].t()) * (h > 0)
        grads[f"A{i}"] = y.t() @ dh
        return dh @ w[f"A{i}"].t(), dr

    def forward(self, tokens):
        """The hidden states for the head, and what the backward needs."""
        w, kept = self.w, []
        x = molt.token_embedding(w["W"], tokens, scale=self.scale)
        s = molt.residual_norm_fwd(x, w_pre=w["norm0"], residual_dtype=F32)
        kept.append((x, None, None, s))
        for i in range(self.blocks):
            s, k = self.block_fwd(i, s)
            kept.append(k)
        return s["y"], kept

    def step(self, tokens, targets, label_smoothing=0.0, z_loss=0.0):
        """Loss and the gradients of all parameters (fp32; the blocks' matrices bf16)."""
        w, grads = self.w, {}
        y, kept = self.forward(tokens)
        out = molt.cross_entropy_fwd_bwd(y, w["W"], targets, label_smoothing=label_smoothing, z_loss=z_loss)
        dy, dr = out["dhidden"], None
        for i in reversed(range(self.blocks)):
            dy, dr = self.block_bwd(i, kept[i + 1], dy, dr, grads)
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


class GatedPolicy(Policy):
    """With blocks of a gated linear recurrence and a gated feed-forward block.  cu_seqlens: the
    sequences among the tokens (None: one).  A forward draws its masks from (seed, draw); set
    `draw` anew for each, p = 0 to leave dropout out."""

    def __init__(self, V, H, blocks, device="cuda", seed=0, p=0.1):
        self.seed, self.draw, self.drop, self.cu_seqlens = seed, 0, p, None
        super().__init__(V, H, blocks, device, seed)

    def make_block(self, i, H, normal, device):
        self.p[f"G{i}"] = normal(H, 2 * H, std=H ** -0.5)
        for name in ("Wg", "Wu"):
            self.p[f"{name}{i}"] = normal(2 * H, H, std=H ** -0.5)
        self.p[f"Wd{i}"] = normal(H, 2 * H, std=(2 * H) ** -0.5)
        for name in (f"mid{i}", f"norm{i + 1}"):
            self.p[name] = torch.ones(H, device=device)

    def masks(self, i):
        """Arguments of dropout for a block's two."""
        return [dict(p=self.drop, seed=self.seed, offset=(self.draw * self.blocks + i) * 2 + j) for j in range(2)]

    def block_fwd(self, i, s):
        w, H, y = self.w, self.H, s["y"]
        m1, m2 = self.masks(i)
        fv = y @ w[f"G{i}"]
        h = molt.gated_scan_fwd(fv[:, :H], fv[:, H:], cu_seqlens=self.cu_seqlens, want_states=True)
        o1 = molt.dropout_fwd(h["y"], **m1)
        s1 = molt.residual_norm_fwd(o1, s["residual"], w_pre=w[f"mid{i}"])
        f = molt.gated_ffn_fwd(s1["y"], w[f"Wg{i}"], w[f"Wu{i}"], w[f"Wd{i}"], keep=True)
        o2 = molt.dropout_fwd(f["y"], **m2)
        s2 = molt.residual_norm_fwd(o2, s1["residual"], w_pre=w[f"norm{i + 1}"])
        return s2, (y, fv, h["states"], o1, s1, f, o2, s2, (m1, m2))

    def block_bwd(self, i, kept, dy, dr, grads):
        w, H = self.w, self.H
        y, fv, states, o1, s1, f, o2, s2, (m1, m2) = kept
        b = molt.residual_norm_bwd(dy, dr, o2, s2["residual"], s2["rstd_pre"], w_pre=w[f"norm{i + 1}"])
        grads[f"norm{i + 1}"] = b["dw_pre"]
        g = molt.gated_ffn_bwd(molt.dropout_bwd(b["dx"], **m2), s1["y"], w[f"Wg{i}"], w[f"Wu{i}"], w[f"Wd{i}"], f["gate"], f["up"])
        grads[f"Wg{i}"], grads[f"Wu{i}"], grads[f"Wd{i}"] = g["dw_gate"], g["dw_up"], g["dw_down"]
        b = molt.residual_norm_bwd(g["dx"], b["dresidual"], o1, s1["residual"], s1["rstd_pre"], w_pre=w[f"mid{i}"])
        grads[f"mid{i}"] = b["dw_pre"]
        g = molt.gated_scan_bwd(molt.dropout_bwd(b["dx"], **m1), fv[:, :H], fv[:, H:], states, cu_seqlens=self.cu_seqlens)
        dfv = torch.cat((g["dgate"], g["dvalue"]), 1)
        grads[f"G{i}"] = y.t() @ dfv
        return dfv @ w[f"G{i}"].t(), b["dresidual"]

    def decode(self, tokens, states):
        """Hidden states of the next token of each sequence, without dropout; `states`, a [B, H] of
        zeros for each block before the first token, are brought up to date."""
        w, H = self.w, self.H
        s = molt.residual_norm_fwd(molt.token_embedding(w["W"], tokens, scale=self.scale), w_pre=w["norm0"], residual_dtype=F32)
        for i, state in enumerate(states):
            fv = s["y"] @ w[f"G{i}"]
            h = molt.gated_scan_step(fv[:, :H], fv[:, H:], state, out_state=state)
            s = molt.residual_norm_fwd(h["y"], s["residual"], w_pre=w[f"mid{i}"])
            f = molt.gated_ffn_fwd(s["y"], w[f"Wg{i}"], w[f"Wu{i}"], w[f"Wd{i}"])
            s = molt.residual_norm_fwd(f["y"], s["residual"], w_pre=w[f"norm{i + 1}"])
        return s["y"]


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
    ap.add_argument("--block", choices=("relu", "gated"), default="relu")
    ap.add_argument("--length", type=int, default=512)
    ap.add_argument("--dropout", type=float, default=0.1)
    a = ap.parse_args(argv)
    if a.length < 1 or not 0 <= a.dropout < 1:
        ap.error("--length is at least 1, --dropout in [0, 1)")
    if a.vocab < 64 or a.hidden % 64:
        ap.error("--vocab is at least 64, --hidden a multiple of 64")
    gated = a.block == "gated"
    policy, state = GatedPolicy(a.vocab, a.hidden, a.blocks, p=a.dropout) if gated else Policy(a.vocab, a.hidden, a.blocks), {}
    if gated:
        policy.cu_seqlens = torch.tensor([*range(0, a.tokens, a.length), a.tokens], dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    losses = []
    for i in range(a.steps):
        tokens, targets = batch(a.tokens, a.vocab, gen)
        if gated:
            policy.draw = i
        loss, grads = policy.step(tokens, targets)
        policy.update(grads, state, a.lr)
        losses.append(float(loss))
        if i % 10 == 0 or i == a.steps - 1:
            print(f"step {i:4d}  loss {losses[-1]:.4f}")
    # the same hidden states in the policy update's forward
    tokens, targets = batch(a.tokens, a.vocab, gen)
    if gated:
        policy.drop = 0.0
    y, _ = policy.forward(tokens)
    out = molt.cross_entropy_fwd(y, policy.w["W"], targets)
    mask = (targets != -100).to(torch.uint8)
    logp, _ = molt.token_logprobs(y, policy.w["W"], targets, mask)
    print(f"held out  loss {float(out['loss']):.4f}  from token_logprobs {-float(logp.double().sum() / mask.sum()):.4f}")
    if gated:
        n = min(a.length, a.tokens)
        states = [torch.zeros(1, a.hidden, device="cuda") for _ in range(a.blocks)]
        steps = torch.cat([policy.decode(tokens[i:i + 1], states) for i in range(n)]).float()
        print(f"{n} tokens decoded  hidden states differ by {float((steps - y[:n].float()).norm() / steps.norm()):.1e}")
    return losses, float(out["loss"])


if __name__ == "__main__":
    main()
