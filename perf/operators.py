"""The operators around the LM head on the residual stream, as measurable cases.

A training step runs them in a row: token ids enter the residual stream
(`token_embedding`), every block hands its output back through a norm, a gate and a
scaled residual and reads the stream through the next norm (`residual_norm_*`), and
the LM head turns the last hidden states into the loss of the next token without
keeping the logits (`cross_entropy_*`); then the same in reverse.  `listed` holds
cases over the range of sizes, `draw` further ones of the same ranges, `run` one
call in its plain form (`own` false: elementary torch operations in 32 bits, rounded
once) or through the library (`own` true).

Inputs are drawn on the device from the seed alone.  Token ids follow Zipf's law (a
few ids make up a tenth of a text), activations have a few outlier channels, half
of the targets are tokens that the hidden state already predicts, and ignored
targets come in spans, as prompts do.
"""
import math

import torch

own = False

H_CHOICES = (256, 320, 512, 896, 1024, 1536, 2048, 2560, 3584, 4096, 5120)
T_MAX, V_MIN, V_MAX = 65536, 1000, 151936
ROWS_LARGEST = 65536 * 4096             # T H of the largest call on rows
HEAD_LARGEST = 8192 * 4096 * 151936     # T H V of the largest call on the LM head
LOGITS_LARGEST = 1 << 32                # T V up to which the plain form's 32-bit logits fit comfortably
EXACT_FLOPS = 4e12                      # fp64 work up to which `exact` computes a case
IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one decoding step of 64 sequences: launch-bound
        {"name": "embed decode step", "kind": "embed", "T": 64, "H": 2048, "V": 32000, "dtype": "bf16", "out": "bf16",
         "scale": 1.0},
        # a whole training window enters the residual stream, scaled by sqrt(H)
        {"name": "embed window", "kind": "embed", "T": 65536, "H": 4096, "V": 151936, "dtype": "bf16", "out": "bf16",
         "scale": 64.0},
        # a ragged microbatch of a small model with fp32 weights; padding carries no gradient
        {"name": "embed gradient ragged", "kind": "embed_bwd", "T": 5003, "H": 320, "V": 50257, "dtype": "fp32",
         "out": "fp32", "scale": 1.0, "padding": 0.1},
        # the window's gradient: as many tokens as half the vocabulary, most rows of dE still zero
        {"name": "embed gradient window", "kind": "embed_bwd", "T": 65536, "H": 4096, "V": 151936, "dtype": "bf16",
         "out": "bf16", "scale": 64.0, "padding": 0.0},
        # one token of one sequence between two blocks while decoding
        {"name": "norm one token", "kind": "norm", "T": 1, "H": 4096, "dtype": "bf16", "res": "bf16", "params": "same",
         "post": True, "gate": "none", "alpha": 1.0, "offset": 1.0},
        # a microbatch with the residual stream in 32 bits and a learned gate per channel
        {"name": "norm mid", "kind": "norm", "T": 32768, "H": 2048, "dtype": "bf16", "res": "fp32", "params": "fp32",
         "post": True, "gate": "channel", "alpha": 0.7071, "offset": 0.0},
        # a small ragged batch, fp16, with a gate for every element
        {"name": "norm gradient ragged", "kind": "norm_bwd", "T": 1031, "H": 896, "dtype": "fp16", "res": "fp16",
         "params": "fp32", "post": False, "gate": "full", "alpha": 1.0, "offset": 0.0},
        # the widest model's microbatch, both norms and the channel gate
        {"name": "norm gradient h5120", "kind": "norm_bwd", "T": 16001, "H": 5120, "dtype": "bf16", "res": "bf16",
         "params": "same", "post": True, "gate": "channel", "alpha": 1.0, "offset": 0.0},
        # evaluation of one short response: W is read once, almost nothing else
        {"name": "cross entropy one response", "kind": "ce_fwd", "T": 100, "H": 4096, "V": 151936, "masked": 0.0,
         "smoothing": 0.0, "z_loss": 0.0, "weights": False},
        # the smallest configuration's step: launch-bound
        {"name": "cross entropy tiny", "kind": "ce", "T": 512, "H": 256, "V": 4096, "masked": 0.2, "smoothing": 0.0,
         "z_loss": 0.0, "weights": False},
        # the mid model with every term of the loss: label smoothing, z term, token weights
        {"name": "cross entropy mid", "kind": "ce", "T": 8192, "H": 2048, "V": 32000, "masked": 0.2, "smoothing": 0.1,
         "z_loss": 1e-4, "weights": True},
        # the large vocabulary, prompts ignored
        {"name": "cross entropy large vocab", "kind": "ce", "T": 8192, "H": 4096, "V": 151936, "masked": 0.3,
         "smoothing": 0.0, "z_loss": 0.0, "weights": False},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("embed", "embed_bwd", "norm", "norm", "norm_bwd", "norm_bwd", "ce_fwd", "ce", "ce"))
    if kind in ("ce_fwd", "ce"):
        while True:
            T, H, V = _log_uniform(rng, 16, T_MAX), rng.choice(H_CHOICES), _log_uniform(rng, V_MIN, V_MAX)
            if T * H * V <= HEAD_LARGEST // 2 and T * V <= LOGITS_LARGEST:
                break
        return {"kind": kind, "T": T, "H": H, "V": V, "masked": round(rng.uniform(0.0, 0.5), 3),
                "smoothing": rng.choice((0.0, 0.0, 0.1)), "z_loss": rng.choice((0.0, 0.0, 1e-4)),
                "weights": rng.random() < 0.3}
    while True:
        T = _log_uniform(rng, 1, T_MAX)
        H = rng.choice(H_CHOICES) if rng.random() < 0.6 else _log_uniform(rng, 64, 5120)
        if T * H <= ROWS_LARGEST and H != 3072:
            break
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if kind in ("embed", "embed_bwd"):
        wide = rng.random() < 0.3
        return {"kind": kind, "T": T, "H": H, "V": _log_uniform(rng, V_MIN, V_MAX), "dtype": dtype,
                "out": "fp32" if wide else dtype, "scale": rng.choice((1.0, round(math.sqrt(H), 4))),
                "padding": rng.choice((0.0, 0.2)) if kind == "embed_bwd" else 0.0}
    return {"kind": kind, "T": T, "H": H, "dtype": dtype, "res": rng.choice((dtype, "fp32")),
            "params": rng.choice(("same", "fp32")), "post": rng.random() < 0.5,
            "gate": rng.choice(("none", "channel", "token", "full")), "alpha": rng.choice((1.0, 0.7071)),
            "offset": rng.choice((0.0, 1.0))}


# ------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _uniform(gen, *shape):
    return torch.rand(*shape, device="cuda", generator=gen)


def _activations(gen, T, H, dtype, scale=1.0):
    """N(0, scale) with every 64th channel or so ten times as large."""
    channel = torch.where(_uniform(gen, H) < 1.0 / 64, 10.0, 1.0) * scale
    return (_normal(gen, T, H) * channel).to(dtype)


def _zipf(gen, T, V):
    """Token ids of frequency 1 / rank, the ranks spread over the vocabulary."""
    rank = (torch.exp(_uniform(gen, T).double() * math.log(V + 1.0)) - 1.0).long().clamp_(0, V - 1)
    return torch.randperm(V, device="cuda", generator=gen)[rank].to(torch.int32)


def _spans(gen, T, frac):
    """Truth values, spans of 64 tokens (fewer in a short batch) of which about `frac` are set."""
    n = max(1, min(64, T // 8))
    hit = _uniform(gen, (T + n - 1) // n) < frac
    hit[0] = False
    return hit.repeat_interleave(n)[:T]


def _prepare_embed(case, gen):
    T, H, V, dtype = case["T"], case["H"], case["V"], DTYPES[case["dtype"]]
    s = {"case": case, "tokens": _zipf(gen, T, V)}
    if case["kind"] == "embed":
        s["weight"] = (_normal(gen, V, H) * 0.02).to(dtype)
        return s
    s["padding"] = 0 if case["padding"] else None
    s["tokens"][_spans(gen, T, case["padding"])] = 0
    s["dout"] = _activations(gen, T, H, dtype, 1e-3)
    return s


def _prepare_norm(case, gen):
    T, H, dtype, res = case["T"], case["H"], DTYPES[case["dtype"]], DTYPES[case["res"]]
    params = dtype if case["params"] == "same" else torch.float32
    weight = lambda: (1.0 - case["offset"] + 0.1 * _normal(gen, H)).to(params)
    s = {"case": case, "eps": 1e-6, "x": _activations(gen, T, H, dtype), "residual": _activations(gen, T, H, res, 3.0),
         "w_pre": weight(), "w_post": weight() if case["post"] else None, "gate": None}
    if case["gate"] == "channel":
        s["gate"] = (0.1 + 0.05 * _normal(gen, H)).to(params)
    elif case["gate"] == "token":
        s["gate"] = _uniform(gen, T)
    elif case["gate"] == "full":
        s["gate"] = torch.sigmoid(_normal(gen, T, H)).to(dtype)
    if case["kind"] == "norm":
        return s
    # what the forward pass has kept
    y, r, rstd_post, rstd_pre = _norm(s, torch.float32)
    s.update(residual=r.to(res), rstd_post=rstd_post, rstd_pre=rstd_pre,
             dy=_activations(gen, T, H, dtype, 1e-3), dresidual=_activations(gen, T, H, res, 1e-3))
    return s


def _prepare_head(case, gen):
    T, H, V = case["T"], case["H"], case["V"]
    W = torch.empty(V, H, device="cuda", dtype=torch.bfloat16).normal_(0.0, 0.02, generator=gen)
    x = _zipf(gen, T, V)
    # the hidden states of every other token or so already point at its target: about 8 above the other logits
    known = (_uniform(gen, T) < 0.5).float() * (8.0 / (H * 4e-4))
    h = (_normal(gen, T, H) + known[:, None] * W[x.long()].float()).to(torch.bfloat16)
    x[_spans(gen, T, case["masked"])] = IGNORE
    return {"case": case, "h": h, "W": W, "x": x,
            "weights": 0.25 + 1.5 * _uniform(gen, T) if case["weights"] else None}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if case["kind"] in ("embed", "embed_bwd"):
        return _prepare_embed(case, gen)
    if case["kind"] in ("norm", "norm_bwd"):
        return _prepare_norm(case, gen)
    return _prepare_head(case, gen)


# -------------------------------------------------------------- plain forms
def _embed(s):
    return (s["weight"][s["tokens"].long()].float() * s["case"]["scale"]).to(DTYPES[s["case"]["out"]])


def _embed_bwd(s):
    case = s["case"]
    ids = s["tokens"].long()
    rows = s["dout"].float() * case["scale"]
    if s["padding"] is not None:
        rows = rows * (ids != s["padding"])[:, None]
    dW = torch.zeros(case["V"], case["H"], device="cuda").index_add_(0, ids, rows)
    return dW.to(DTYPES[case["out"]])


def _gate(s, wide):
    g = s["gate"].to(wide)
    return g[:, None] if s["case"]["gate"] == "token" else g


def _norm(s, wide):
    """(y, residual, rstd_post, rstd_pre) in the type `wide`."""
    case = s["case"]
    u, rstd_post = s["x"].to(wide), None
    if s["w_post"] is not None:
        rstd_post = torch.rsqrt((u * u).mean(1) + s["eps"])
        u = u * rstd_post[:, None] * (case["offset"] + s["w_post"].to(wide))
    if s["gate"] is not None:
        u = u * _gate(s, wide)
    r = case["alpha"] * s["residual"].to(wide) + u
    rstd_pre = torch.rsqrt((r * r).mean(1) + s["eps"])
    return r * rstd_pre[:, None] * (case["offset"] + s["w_pre"].to(wide)), r, rstd_post, rstd_pre


def _norm_bwd(s, wide):
    """The gradients in the type `wide`, as run's dict lays them out."""
    case = s["case"]
    dy, r = s["dy"].to(wide), s["residual"].to(wide)
    xh = r * s["rstd_pre"].to(wide)[:, None]
    q = dy * (case["offset"] + s["w_pre"].to(wide))
    D = s["dresidual"].to(wide) + s["rstd_pre"].to(wide)[:, None] * (q - xh * (q * xh).mean(1, keepdim=True))
    out = {"dresidual": case["alpha"] * D, "dw_pre": (dy * xh).sum(0), "dw_post": None, "dgate": None}
    a = s["x"].to(wide)
    ah = a if s["w_post"] is None else a * s["rstd_post"].to(wide)[:, None]
    w = None if s["w_post"] is None else case["offset"] + s["w_post"].to(wide)
    du = D
    if s["gate"] is not None:
        du = D * _gate(s, wide)
        Du = D * (ah if w is None else ah * w)
        out["dgate"] = {"channel": lambda: Du.sum(0), "token": lambda: Du.sum(1), "full": lambda: Du}[case["gate"]]()
    if w is None:
        out["dx"] = du
        return out
    out["dw_post"] = (du * ah).sum(0)
    p = du * w
    out["dx"] = s["rstd_post"].to(wide)[:, None] * (p - ah * (p * ah).mean(1, keepdim=True))
    return out


def _norm_bwd_rounded(s):
    case = s["case"]
    out = _norm_bwd(s, torch.float32)
    out["dx"] = out["dx"].to(DTYPES[case["dtype"]])
    out["dresidual"] = out["dresidual"].to(DTYPES[case["res"]])
    if case["gate"] == "full":
        out["dgate"] = out["dgate"].to(DTYPES[case["dtype"]])
    return out


def _head(s, wide, grad):
    """Loss, log-probs, lse and, with `grad`, dhidden and dW in the type `wide`."""
    case = s["case"]
    eps, zc, V = case["smoothing"], case["z_loss"], case["V"]
    h, W = s["h"].to(wide), s["W"].to(wide)
    act = s["x"] != IGNORE
    x = torch.where(act, s["x"], torch.zeros_like(s["x"])).long()
    z = h @ W.t()
    top = z.max(1, keepdim=True).values
    lse = top[:, 0] + torch.log(torch.exp(z - top).sum(1))
    logp = z.gather(1, x[:, None])[:, 0] - lse
    l = -(1.0 - eps) * logp + zc * lse * lse
    if eps:
        l = l + eps * (lse - z.mean(1))
    c = act.to(wide) / act.sum()
    if s["weights"] is not None:
        c = c * s["weights"].to(wide)
    zero = torch.zeros_like(lse)
    out = {"loss": (l * c).sum().reshape(1), "logp": torch.where(act, logp, zero), "lse": torch.where(act, lse, zero)}
    if not grad:
        return out
    g = z.sub_(lse[:, None]).exp_().mul_((c * (1.0 + 2.0 * zc * lse))[:, None])
    if eps:
        g.sub_((c * (eps / V))[:, None])
    g.scatter_add_(1, x[:, None], -((1.0 - eps) * c)[:, None])
    out["dhidden"] = g @ W
    out["dW"] = g.t() @ h
    return out


def _head_rounded(s, grad):
    out = _head(s, torch.float32, grad)
    if grad:
        out["dhidden"], out["dW"] = out["dhidden"].to(torch.bfloat16), out["dW"].to(torch.bfloat16)
    return out


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "embed":
        return _embed(s)
    if kind == "embed_bwd":
        return _embed_bwd(s)
    if kind == "norm":
        y, r, rstd_post, rstd_pre = _norm(s, torch.float32)
        return {"y": y.to(DTYPES[s["case"]["dtype"]]), "residual": r.to(DTYPES[s["case"]["res"]]),
                "rstd_post": rstd_post, "rstd_pre": rstd_pre}
    if kind == "norm_bwd":
        return _norm_bwd_rounded(s)
    return _head_rounded(s, kind == "ce")


# ------------------------------------------------------- the library's calls
def _run_own(s):
    import paper_2607_21653_gb300 as molt
    case = s["case"]
    kind = case["kind"]
    if kind == "embed":
        return molt.token_embedding(s["weight"], s["tokens"], scale=case["scale"], out_dtype=DTYPES[case["out"]])
    if kind == "embed_bwd":
        return molt.token_embedding_bwd(s["dout"], s["tokens"], case["V"], scale=case["scale"],
                                        padding_idx=s["padding"], dtype=DTYPES[case["out"]])
    if kind == "norm":
        return molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"],
                                      res_scale=case["alpha"], eps=s["eps"], weight_offset=case["offset"])
    if kind == "norm_bwd":
        return molt.residual_norm_bwd(s["dy"], s["dresidual"], s["x"], s["residual"], s["rstd_pre"],
                                      rstd_post=s["rstd_post"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"],
                                      res_scale=case["alpha"], weight_offset=case["offset"])
    if kind == "ce_fwd":
        out = molt.cross_entropy_fwd(s["h"], s["W"], s["x"], ignore_index=IGNORE, token_weight=s["weights"],
                                     label_smoothing=case["smoothing"], z_loss=case["z_loss"])
    else:
        out = molt.cross_entropy_fwd_bwd(s["h"], s["W"], s["x"], ignore_index=IGNORE, token_weight=s["weights"],
                                         label_smoothing=case["smoothing"], z_loss=case["z_loss"],
                                         dW_dtype=torch.bfloat16)
    out.pop("stats")
    return out


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ----------------------------------------------------------------- measures
def work(case):
    kind, T, H = case["kind"], case["T"], case["H"]
    if kind in ("ce_fwd", "ce"):
        V = case["V"]
        act = T * (1.0 - case["masked"])
        read = act * H * 2 + V * H * 2 + T * 4
        if kind == "ce_fwd":
            return {"bytes": read + T * 8, "flops": 2.0 * act * H * V}
        return {"bytes": read + T * 8 + T * H * 2 + V * H * 2, "flops": 6.0 * act * H * V}
    b = BYTES[case["dtype"]]
    if kind == "embed":
        # distinct ids of a Zipf text of T tokens: each rank r is met with probability 1 - (1 - 1 / (r ln V))^T
        lnV = math.log(case["V"] + 1.0)
        met = min(T, case["V"], int(T / lnV * (1.0 + math.log(max(1.0, case["V"] * lnV / T)))) + 1)
        return {"bytes": T * 4 + met * H * b + T * H * BYTES[case["out"]], "flops": 1.0 * T * H}
    if kind == "embed_bwd":
        return {"bytes": T * 4 + T * H * b * (1.0 - case["padding"]) + case["V"] * H * BYTES[case["out"]],
                "flops": 1.0 * T * H}
    r = BYTES[case["res"]]
    gate = T * H * b if case["gate"] == "full" else 0
    if kind == "norm":
        return {"bytes": T * H * (2 * b + 2 * r) + gate, "flops": 12.0 * T * H}
    return {"bytes": T * H * (3 * b + 3 * r) + 2 * gate, "flops": 30.0 * T * H}


# ----------------------------------------------------------------- 64 bits
def _exact_embed_bwd(s):
    """Sums of the rows of equal tokens, from prefix sums over the sorted tokens a piece of columns at a time."""
    case = s["case"]
    ids, order = torch.sort(s["tokens"].long(), stable=True)
    d = s["dout"].double()
    out = torch.zeros(case["V"], case["H"], device="cuda", dtype=torch.float64)
    last = torch.ones_like(ids, dtype=torch.bool)
    last[:-1] = ids[1:] != ids[:-1]
    ends = last.nonzero()[:, 0]
    for a in range(0, case["H"], 512):
        total = torch.cumsum(d[order, a:a + 512], 0)[ends]
        total[1:] -= total[:-1].clone()
        out[ids[ends], a:a + 512] = total * case["scale"]
    if s["padding"] is not None:
        out[s["padding"]] = 0.0
    return out


def _exact_norm(s):
    case, d = s["case"], torch.float64
    a, r, g = s["x"].to(d), s["residual"].to(d), s["gate"]
    out = {"rstd_post": None}
    if s["w_post"] is not None:
        ms = (a ** 2).sum(1) / case["H"] + s["eps"]
        out["rstd_post"] = 1.0 / ms.sqrt()
        a = a / ms.sqrt()[:, None] * (s["w_post"].to(d) + case["offset"])
    if g is not None:
        a = a * (g.to(d)[:, None] if case["gate"] == "token" else g.to(d))
    t = r * case["alpha"] + a
    ms = (t ** 2).sum(1) / case["H"] + s["eps"]
    return {"y": t / ms.sqrt()[:, None] * (s["w_pre"].to(d) + case["offset"]), "residual": t,
            "rstd_post": out["rstd_post"], "rstd_pre": 1.0 / ms.sqrt()}


def _exact_norm_bwd(s):
    """By the Jacobians: y_i = w_i n_i with dn_i / dr_j = rstd ([i = j] - n_i n_j / H)."""
    case, d = s["case"], torch.float64

    def through(rstd, n, w, up):   # (gradient of the input, of the weight) of w n, n = rstd v
        v = up * w
        return rstd[:, None] * (v - n * (torch.einsum("th,th->t", v, n) / case["H"])[:, None]), \
            torch.einsum("th,th->h", up, n)

    rstd = s["rstd_pre"].to(d)
    back, dw_pre = through(rstd, s["residual"].to(d) * rstd[:, None], s["w_pre"].to(d) + case["offset"], s["dy"].to(d))
    D = s["dresidual"].to(d) + back
    a, g, w_post = s["x"].to(d), s["gate"], None
    n = u = a
    if s["w_post"] is not None:
        w_post = s["w_post"].to(d) + case["offset"]
        n = a * s["rstd_post"].to(d)[:, None]
        u = n * w_post
    dgate, du = None, D
    if g is not None:
        du = D * (g.to(d)[:, None] if case["gate"] == "token" else g.to(d))
        dgate = {"channel": "th,th->h", "token": "th,th->t", "full": "th,th->th"}[case["gate"]]
        dgate = torch.einsum(dgate, D, u)
    dw_post = None
    if w_post is not None:
        du, dw_post = through(s["rstd_post"].to(d), n, w_post, du)
    return {"dresidual": D * case["alpha"], "dw_pre": dw_pre, "dw_post": dw_post, "dgate": dgate, "dx": du}


def _exact_head(s, grad):
    """Over the active rows alone, a piece of them at a time."""
    case, d = s["case"], torch.float64
    T, V, e, zc = case["T"], case["V"], case["smoothing"], case["z_loss"]
    W = s["W"].to(d)
    rows = (s["x"] != IGNORE).nonzero()[:, 0]
    n = rows.numel()
    out = {"loss": torch.zeros(1, device="cuda", dtype=d), "logp": torch.zeros(T, device="cuda", dtype=d),
           "lse": torch.zeros(T, device="cuda", dtype=d)}
    if grad:
        out["dhidden"], out["dW"] = torch.zeros_like(s["h"], dtype=d), torch.zeros_like(W)
    step = max(1, (1 << 27) // V)
    for a in range(0, n, step):
        k = rows[a:a + step]
        h = s["h"][k].to(d)
        q = torch.zeros(k.numel(), V, device="cuda", dtype=d).scatter_(1, s["x"][k].long()[:, None], 1.0)
        z = h @ W.t()
        lse = torch.logsumexp(z, 1)
        out["lse"][k], out["logp"][k] = lse, (z * q).sum(1) - lse
        q = q * (1.0 - e) + e / V                       # the smoothed target distribution
        w = torch.ones(k.numel(), device="cuda", dtype=d) if s["weights"] is None else s["weights"][k].to(d)
        out["loss"] += (w * (lse - (q * z).sum(1) + zc * lse ** 2)).sum() / n
        if grad:
            g = (torch.softmax(z, 1) * (1.0 + 2.0 * zc * lse)[:, None] - q) * (w / n)[:, None]
            out["dhidden"][k] = g @ W
            out["dW"].addmm_(g.t(), h)
    return out


def exact(case, seed):
    kind = case["kind"]
    if kind in ("ce_fwd", "ce") and work(case)["flops"] > EXACT_FLOPS:
        return None
    s = prepare(case, seed)
    if kind == "embed":
        return torch.index_select(s["weight"], 0, s["tokens"]).double() * case["scale"]
    if kind == "embed_bwd":
        return _exact_embed_bwd(s)
    if kind == "norm":
        return _exact_norm(s)
    if kind == "norm_bwd":
        return _exact_norm_bwd(s)
    return _exact_head(s, kind == "ce")
