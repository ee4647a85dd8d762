"""The operators inside a block, as measurable cases.

Between two norms of the residual stream a block mixes tokens or channels and drops
part of the result: the gated linear recurrence over packed sequences (`gated_scan_*`,
with its step for one token of each sequence), the gated feed-forward block
(`gated_ffn_*`) and dropout from a counter, whose mask is never stored (`dropout_*`).
`listed` holds cases over the range of sizes, `draw` further ones of the same ranges,
`run` one call in its plain form (`own` false: elementary torch operations in 32 bits,
rounded once) or through the library (`own` true).

Inputs are drawn on the device from the seed alone.  Activations have a few outlier
channels, channels of the recurrence remember from a few tokens to a few hundred, and
sequences of a packed batch are of uneven lengths, some of them empty.
"""
import math

import torch

own = False

H_CHOICES = (256, 320, 512, 896, 1024, 1536, 2048, 2560, 3584, 4096, 5120)
T_MAX_FFN, T_MAX_ROWS = 16384, 65536
F_MAX = 12288
FFN_LARGEST = 16384 * 4096 * 10944      # T H F of the largest feed-forward call
ROWS_LARGEST = 65536 * 4096             # T H of the largest call on rows
CHECKPOINT = 128                        # rows between the states that a scan's forward keeps for its backward
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # one token of one sequence: nothing but the three weights to read
        {"name": "ffn one token", "kind": "ffn", "T": 1, "H": 4096, "F": 10944, "dtype": "bf16", "act": "silu",
         "keep": False},
        # a ragged microbatch of a small model in its forward pass, gate and up kept for the backward
        {"name": "ffn ragged", "kind": "ffn", "T": 1031, "H": 896, "F": 2392, "dtype": "fp16", "act": "gelu",
         "keep": True},
        # a whole training window
        {"name": "ffn window", "kind": "ffn", "T": 16384, "H": 4096, "F": 10944, "dtype": "bf16", "act": "silu",
         "keep": True},
        # the small model's backward pass
        {"name": "ffn gradient ragged", "kind": "ffn_bwd", "T": 1031, "H": 896, "F": 2392, "dtype": "fp16",
         "act": "gelu", "kept": True},
        # half a window's backward pass, gate and up formed again in the place of being kept
        {"name": "ffn gradient", "kind": "ffn_bwd", "T": 8192, "H": 4096, "F": 10944, "dtype": "bf16", "act": "silu",
         "kept": False},
        # one decoding step of 64 sequences
        {"name": "scan step", "kind": "scan_step", "B": 64, "H": 4096, "dtype": "bf16", "form": "sigmoid"},
        # a window of four long trajectories, its states kept
        {"name": "scan window", "kind": "scan", "T": 65536, "H": 4096, "B": 4, "dtype": "bf16", "form": "sigmoid",
         "initial": False},
        # a ragged microbatch in 32 bits whose sequences go on from earlier segments
        {"name": "scan gradient ragged", "kind": "scan_bwd", "T": 5003, "H": 320, "B": 13, "dtype": "fp32",
         "form": "log", "initial": True},
        # the backward pass of one long trajectory
        {"name": "scan gradient long", "kind": "scan_bwd", "T": 32768, "H": 2048, "B": 1, "dtype": "bf16",
         "form": "sigmoid", "initial": False},
        # a small model's microbatch
        {"name": "dropout small", "kind": "dropout", "T": 512, "H": 256, "dtype": "bf16", "res": "none", "p": 0.1},
        # a window's block output into a residual stream in 32 bits
        {"name": "dropout window", "kind": "dropout", "T": 32768, "H": 4096, "dtype": "bf16", "res": "fp32", "p": 0.1},
        # its backward pass at the widest model
        {"name": "dropout gradient", "kind": "dropout_bwd", "T": 16001, "H": 5120, "dtype": "bf16", "res": "none",
         "p": 0.25},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("ffn", "ffn", "ffn_bwd", "ffn_bwd", "scan", "scan", "scan_bwd", "scan_bwd", "scan_step", "dropout",
                       "dropout_bwd"))
    if kind in ("ffn", "ffn_bwd"):
        while True:
            T = _log_uniform(rng, 1, T_MAX_FFN)
            H = rng.choice(H_CHOICES) if rng.random() < 0.6 else 8 * _log_uniform(rng, 8, 640)
            F = 8 * _log_uniform(rng, 8, F_MAX // 8)
            if T * H * F <= FFN_LARGEST // (2 if kind == "ffn" else 4):
                break
        case = {"kind": kind, "T": T, "H": H, "F": F, "dtype": rng.choice(("bf16", "bf16", "fp16")),
                "act": rng.choice(("silu", "silu", "gelu", "relu"))}
        case["keep" if kind == "ffn" else "kept"] = rng.random() < 0.5
        return case
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    form = rng.choice(("sigmoid", "log"))
    if kind == "scan_step":
        return {"kind": kind, "B": _log_uniform(rng, 1, 1024), "H": _log_uniform(rng, 64, 5120), "dtype": dtype,
                "form": form}
    while True:
        T = _log_uniform(rng, 1, T_MAX_ROWS)
        H = rng.choice(H_CHOICES) if rng.random() < 0.6 else _log_uniform(rng, 64, 5120)
        if T * H <= ROWS_LARGEST // 2:
            break
    if kind in ("scan", "scan_bwd"):
        return {"kind": kind, "T": T, "H": H, "B": _log_uniform(rng, 1, 256), "dtype": dtype, "form": form,
                "initial": rng.random() < 0.5}
    return {"kind": kind, "T": T, "H": H, "dtype": dtype, "res": rng.choice(("none", dtype, "fp32")),
            "p": rng.choice((0.05, 0.1, 0.25, 0.5))}


# ------------------------------------------------------------------- inputs
def _normal(gen, *shape):
    return torch.randn(*shape, device="cuda", generator=gen)


def _uniform(gen, *shape):
    return torch.rand(*shape, device="cuda", generator=gen)


def _activations(gen, T, H, dtype, scale=1.0):
    """N(0, scale) with every 64th channel or so four times as large."""
    channel = torch.where(_uniform(gen, H) < 1.0 / 64, 4.0, 1.0) * scale
    return (_normal(gen, T, H) * channel).to(dtype)


def _prepare_ffn(case, gen):
    T, H, F, dtype = case["T"], case["H"], case["F"], DTYPES[case["dtype"]]
    s = {"case": case, "x": _activations(gen, T, H, dtype), "w_gate": (_normal(gen, F, H) * H**-0.5).to(dtype),
         "w_up": (_normal(gen, F, H) * H**-0.5).to(dtype), "w_down": (_normal(gen, H, F) * F**-0.5).to(dtype)}
    if case["kind"] == "ffn":
        return s
    # a loss scaled as training in 16 bits scales it
    s["dy"] = _activations(gen, T, H, dtype, 0.05)
    s["gate"] = s["up"] = None
    if case["kept"]:
        s["gate"] = (s["x"].float() @ s["w_gate"].float().t()).to(dtype)
        s["up"] = (s["x"].float() @ s["w_up"].float().t()).to(dtype)
    return s


def _logits(case, gen, T):
    """Gates whose channels remember from a few tokens to a few hundred."""
    H, dtype = case["H"], DTYPES[case["dtype"]]
    f = _normal(gen, T, H) + 5.0 * _uniform(gen, H)
    if case["form"] == "log":
        f = torch.log1p(torch.exp(-f)).neg_()
    return f.to(dtype)


def _prepare_scan(case, gen):
    T, H, B, dtype = case["T"], case["H"], case["B"], DTYPES[case["dtype"]]
    cut = torch.sort((_uniform(gen, B - 1) * T).long()).values if B > 1 else torch.empty(0, dtype=torch.long, device="cuda")
    ends = torch.tensor([0, T], device="cuda")
    s = {"case": case, "gate": _logits(case, gen, T), "value": _activations(gen, T, H, dtype),
         "cu": torch.cat([ends[:1], cut, ends[1:]]).to(torch.int32), "h0": _normal(gen, B, H) if case["initial"] else None}
    if case["kind"] == "scan":
        return s
    s["dy"] = _activations(gen, T, H, dtype, 0.05)
    s["dfinal"] = 0.05 * _normal(gen, B, H) if case["initial"] else None
    s["states"] = _states(_scan(s, torch.float32)[0])   # what the forward pass has kept
    return s


def _prepare_step(case, gen):
    B, H, dtype = case["B"], case["H"], DTYPES[case["dtype"]]
    return {"case": case, "gate": _logits(case, gen, B), "value": _activations(gen, B, H, dtype), "state": _normal(gen, B, H)}


def _prepare_dropout(case, gen):
    T, H, dtype = case["T"], case["H"], DTYPES[case["dtype"]]
    words = torch.randint(0, 1 << 40, (2,), device="cuda", generator=gen).tolist()
    res = None if case["res"] == "none" else DTYPES[case["res"]]
    s = {"case": case, "seed": words[0], "offset": words[1], "residual": None}
    if case["kind"] == "dropout":
        s["x"] = _activations(gen, T, H, dtype)
        s["residual"] = None if res is None else _activations(gen, T, H, res, 3.0)
    else:
        s["x"] = _activations(gen, T, H, dtype if res is None else res, 1e-3)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    return {"ffn": _prepare_ffn, "ffn_bwd": _prepare_ffn, "scan": _prepare_scan, "scan_bwd": _prepare_scan,
            "scan_step": _prepare_step, "dropout": _prepare_dropout, "dropout_bwd": _prepare_dropout}[kind](case, gen)


# -------------------------------------------------------------- plain forms
GELU_A, GELU_B = math.sqrt(2.0 / math.pi), 0.044715


def _act(name, g):
    """act(g) and act'(g)."""
    if name == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    p = 1.0 / (1.0 + torch.exp(-2.0 * GELU_A * (g + GELU_B * g * g * g)))   # (1 + tanh) / 2
    return g * p, p + g * p * (1.0 - p) * 2.0 * GELU_A * (1.0 + 3.0 * GELU_B * g * g)


def _ffn(s):
    x, dtype = s["x"].float(), s["x"].dtype
    g, u = x @ s["w_gate"].float().t(), x @ s["w_up"].float().t()
    y = ((_act(s["case"]["act"], g)[0] * u) @ s["w_down"].float().t()).to(dtype)
    keep = s["case"]["keep"]
    return {"y": y, "gate": g.to(dtype) if keep else None, "up": u.to(dtype) if keep else None}


def _ffn_bwd(s):
    dtype = s["x"].dtype
    x, dy, wg, wu, wd = (s[k].float() for k in ("x", "dy", "w_gate", "w_up", "w_down"))
    g = x @ wg.t() if s["gate"] is None else s["gate"].float()
    u = x @ wu.t() if s["up"] is None else s["up"].float()
    a, da = _act(s["case"]["act"], g)
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    return {"dx": (dg @ wg + du @ wu).to(dtype), "dw_gate": (dg.t() @ x).to(dtype), "dw_up": (du.t() @ x).to(dtype),
            "dw_down": (dy.t() @ (a * u)).to(dtype)}


def _decay(s, wide):
    """a and b of h_t = a_t h_{t-1} + b_t, and 1 - a (for the sigmoid form)."""
    f, v = s["gate"].to(wide), s["value"].to(wide)
    if s["case"]["form"] == "log":
        return torch.exp(f), v, None
    na = 1.0 / (1.0 + torch.exp(f))
    return 1.0 / (1.0 + torch.exp(-f)), na * v, na


def _rows_of(s):
    """Of every row: its sequence, whether it is the first one of it, and whether the last."""
    cu, T = s["cu"].long(), s["case"]["T"]
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    return b, t == cu[b], t + 1 == cu[b + 1]


def _linear(a, b, longest):
    """h_t = a_t h_{t-1} + b_t from h_{-1} = 0, by pairs of neighbours, pairs of pairs and so on."""
    a, d = a.clone(), 1
    while d < min(longest, a.shape[0]):
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _scan(s, wide):
    """h of every row, and a, b, 1 - a, the rows' sequences, firsts and lasts."""
    a, b, na = _decay(s, wide)
    seq, first, last = _rows_of(s)
    start = b if s["h0"] is None else b + a * s["h0"].to(wide)[seq]
    h = _linear(torch.where(first[:, None], 0.0, a).to(wide), torch.where(first[:, None], start, b), a.shape[0])
    return h, a, b, na, seq, first, last


def _final(s, h, seq, last):
    out = torch.zeros(s["case"]["B"], s["case"]["H"], device="cuda", dtype=h.dtype)
    if s["h0"] is not None:
        out += s["h0"].to(h.dtype)
    rows = last.nonzero()[:, 0]
    out[seq[rows]] = h[rows]
    return out


def _states(h):
    """The state before every 128th row; zeros before the first."""
    return torch.cat([torch.zeros_like(h[:1]), h[CHECKPOINT - 1:-1:CHECKPOINT]]).float()


def _scan_fwd(s):
    h, _, _, _, seq, _, last = _scan(s, torch.float32)
    return {"y": h.to(s["value"].dtype), "final_state": _final(s, h, seq, last), "states": _states(h)}


def _scan_bwd(s):
    wide = torch.float32
    h, a, _, na, seq, first, last = _scan(s, wide)
    D = s["dy"].to(wide)
    if s["dfinal"] is not None:
        D = torch.where(last[:, None], D + s["dfinal"][seq], D)
    # D_t += a_{t+1} D_{t+1} inside a sequence: the same recurrence, rows backwards
    after = torch.where(last[:, None], 0.0, torch.cat([a[1:], a[:1]]))
    D = _linear(after.flip(0), D.flip(0), a.shape[0]).flip(0)
    before = torch.cat([h[:1], h[:-1]])
    h0 = torch.zeros(case_rows(s), device="cuda") if s["h0"] is None else s["h0"]
    before = torch.where(first[:, None], h0[seq], before)
    out = {"dinitial_state": None}
    if s["h0"] is not None:
        rows = first.nonzero()[:, 0]
        out["dinitial_state"] = s["dfinal"].clone()
        out["dinitial_state"][seq[rows]] = (a * D)[rows]
    if na is None:
        dgate, dvalue = D * before * a, D
    else:
        dgate, dvalue = D * (before - s["value"].to(wide)) * a * na, D * na
    dtype = s["value"].dtype
    return {"dgate": dgate.to(dtype), "dvalue": dvalue.to(dtype), **out}


def case_rows(s):
    return s["case"]["B"], s["case"]["H"]


def _step(s):
    a, b, _ = _decay(s, torch.float32)
    h = a * s["state"] + b
    return {"y": h.to(s["value"].dtype), "state": h}


LOW = (1 << 32) - 1


def _philox(counter, key):
    """Ten rounds on four 32-bit words held in int64 (the low half of a product that wraps is still right)."""
    c0, c1, c2, c3 = counter
    k0, k1 = key
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & LOW) ^ c1 ^ k0, p1 & LOW, ((p0 >> 32) & LOW) ^ c3 ^ k1, p0 & LOW
        k0, k1 = (k0 + 0x9E3779B9) & LOW, (k1 + 0xBB67AE85) & LOW
    return c0, c1, c2, c3


def _threshold(p):
    return int(math.floor(p * 65536.0 + 0.5))


def _kept(s):
    """Truth values [T, H]: 16 bits of the counter (column / 8, row, offset) against p."""
    T, H = s["x"].shape
    col = torch.arange((H + 7) // 8, device="cuda")[None, :]
    row = torch.arange(T, device="cuda")[:, None]
    zero = torch.zeros_like(col + row)
    words = _philox((col + zero, row + zero, zero + (s["offset"] & LOW), zero + (s["offset"] >> 32)),
                    (s["seed"] & LOW, s["seed"] >> 32))
    halves = torch.stack([w >> k & 0xFFFF for w in words for k in (0, 16)], 2)
    return halves.reshape(T, -1)[:, :H] >= _threshold(s["case"]["p"])


def _dropout(s):
    case = s["case"]
    scale = 65536.0 / (65536.0 - _threshold(case["p"]))
    out = torch.where(_kept(s), s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        return (s["residual"].float() + out).to(s["residual"].dtype)
    return out.to(DTYPES[case["dtype"]])


def _run_plain(s):
    return {"ffn": _ffn, "ffn_bwd": _ffn_bwd, "scan": _scan_fwd, "scan_bwd": _scan_bwd, "scan_step": _step,
            "dropout": _dropout, "dropout_bwd": _dropout}[s["case"]["kind"]](s)


# ------------------------------------------------------- the library's calls
def _run_own(s):
    import paper_2607_21653_gb300 as molt
    case = s["case"]
    kind = case["kind"]
    if kind == "ffn":
        return molt.gated_ffn_fwd(s["x"], s["w_gate"], s["w_up"], s["w_down"], activation=case["act"], keep=case["keep"])
    if kind == "ffn_bwd":
        return molt.gated_ffn_bwd(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"], gate=s["gate"], up=s["up"],
                                  activation=case["act"], dw_dtype=s["x"].dtype)
    if kind == "scan":
        return molt.gated_scan_fwd(s["gate"], s["value"], initial_state=s["h0"], cu_seqlens=s["cu"], kind=case["form"],
                                   want_states=True)
    if kind == "scan_bwd":
        return molt.gated_scan_bwd(s["dy"], s["gate"], s["value"], s["states"], initial_state=s["h0"], cu_seqlens=s["cu"],
                                   dfinal_state=s["dfinal"], kind=case["form"])
    if kind == "scan_step":
        return molt.gated_scan_step(s["gate"], s["value"], s["state"], kind=case["form"])
    if kind == "dropout":
        return molt.dropout_fwd(s["x"], case["p"], s["seed"], offset=s["offset"], residual=s["residual"])
    return molt.dropout_bwd(s["x"], case["p"], s["seed"], offset=s["offset"], dtype=DTYPES[case["dtype"]])


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ----------------------------------------------------------------- measures
def work(case):
    kind, H, b = case["kind"], case["H"], BYTES[case["dtype"]]
    if kind in ("ffn", "ffn_bwd"):
        T, F = case["T"], case["F"]
        if kind == "ffn":
            return {"bytes": b * (2 * T * H + 3 * H * F + (2 * T * F if case["keep"] else 0)), "flops": 6.0 * T * H * F}
        return {"bytes": b * (3 * T * H + 6 * H * F + (2 * T * F if case["kept"] else 0)),
                "flops": (12.0 if case["kept"] else 16.0) * T * H * F}
    if kind == "scan_step":
        return {"bytes": case["B"] * H * (3 * b + 8), "flops": 10.0 * case["B"] * H}
    T = case["T"]
    if kind in ("scan", "scan_bwd"):
        ends = case["B"] * H * 4
        kept = (T + CHECKPOINT - 1) // CHECKPOINT * H * 4
        if kind == "scan":
            return {"bytes": 3 * T * H * b + kept + ends * (2 if case["initial"] else 1), "flops": 10.0 * T * H}
        return {"bytes": 5 * T * H * b + kept + ends * (3 if case["initial"] else 0), "flops": 25.0 * T * H}
    r = b if case["res"] == "none" else BYTES[case["res"]]
    if kind == "dropout":
        return {"bytes": T * H * (b + (r if case["res"] == "none" else 2 * r)), "flops": 2.0 * T * H}
    return {"bytes": T * H * (b + r), "flops": 2.0 * T * H}


# ----------------------------------------------------------------- 64 bits
def _exact_ffn(s):
    case, d = s["case"], torch.float64
    x, wg, wu, wd = (s[k].to(d) for k in ("x", "w_gate", "w_up", "w_down"))
    F = torch.nn.functional
    act = {"silu": F.silu, "relu": F.relu, "gelu": lambda t: F.gelu(t, approximate="tanh")}[case["act"]]
    g = torch.einsum("th,fh->tf", x, wg) if s.get("gate") is None else s["gate"].to(d)
    u = torch.einsum("th,fh->tf", x, wu) if s.get("up") is None else s["up"].to(d)
    if case["kind"] == "ffn":
        return {"y": torch.einsum("tf,hf->th", act(g) * u, wd), "gate": g if case["keep"] else None,
                "up": u if case["keep"] else None}
    dy = s["dy"].to(d)
    with torch.enable_grad():
        g, u = g.requires_grad_(), u.requires_grad_()
        h = act(g) * u
    dg, du = torch.autograd.grad(h, (g, u), torch.einsum("th,hf->tf", dy, wd))
    return {"dx": torch.einsum("tf,fh->th", dg, wg) + torch.einsum("tf,fh->th", du, wu),
            "dw_gate": torch.einsum("tf,th->fh", dg, x), "dw_up": torch.einsum("tf,th->fh", du, x),
            "dw_down": torch.einsum("th,tf->hf", dy, h.detach())}


def _exact_scan(s):
    """One row after the other, forwards, and for the gradients backwards."""
    case, d = s["case"], torch.float64
    T, B, H = case["T"], case["B"], case["H"]
    cu = s["cu"].tolist()
    f, v = s["gate"].to(d), s["value"].to(d)
    a = torch.sigmoid(f) if case["form"] == "sigmoid" else torch.exp(f)
    b = torch.sigmoid(-f) * v if case["form"] == "sigmoid" else v
    ends = torch.zeros(B, H, device="cuda", dtype=d) if s["h0"] is None else s["h0"].to(d)
    begin, ends = ends, ends.clone()
    h = torch.empty_like(b)
    for n in range(B):
        at = begin[n]
        for t in range(cu[n], cu[n + 1]):
            at = torch.addcmul(b[t], a[t], at, out=h[t])
        ends[n] = at
    if case["kind"] == "scan":
        kept = torch.zeros((T + CHECKPOINT - 1) // CHECKPOINT, H, device="cuda", dtype=d)
        kept[1:] = h[torch.arange(1, kept.shape[0], device="cuda") * CHECKPOINT - 1]
        return {"y": h, "final_state": ends, "states": kept}
    up = s["dy"].to(d).clone()      # becomes the gradient of h
    back = torch.zeros(B, H, device="cuda", dtype=d) if s["dfinal"] is None else s["dfinal"].to(d).clone()
    for n in range(B):
        for t in range(cu[n + 1] - 1, cu[n] - 1, -1):
            up[t] += back[n]
            torch.mul(a[t], up[t], out=back[n])
    prev = torch.empty_like(h)
    prev[1:] = h[:-1]
    for n in range(B):
        if cu[n] < cu[n + 1]:
            prev[cu[n]] = begin[n]
    da = up * prev
    if case["form"] == "sigmoid":
        dgate, dvalue = (da - up * v) * a * (1.0 - a), up * torch.sigmoid(-f)
    else:
        dgate, dvalue = da * a, up
    return {"dgate": dgate, "dvalue": dvalue, "dinitial_state": None if s["h0"] is None else back}


def _exact_step(s):
    d = torch.float64
    f, v, h = s["gate"].to(d), s["value"].to(d), s["state"].to(d)
    if s["case"]["form"] == "sigmoid":
        h = torch.lerp(v, h, torch.sigmoid(f))
    else:
        h = h * torch.exp(f) + v
    return {"y": h, "state": h}


def _exact_dropout(s):
    """The generator again, its products from halves of 16 bits, on the groups of a piece of rows at a time."""
    case, d = s["case"], torch.float64
    T, H = s["x"].shape
    G = (H + 7) // 8
    keep = torch.empty(T, G * 8, device="cuda", dtype=torch.bool)

    def times(c, m):                # (high, low) words of c m
        cl, ch, ml, mh = c & 0xFFFF, c >> 16, m & 0xFFFF, m >> 16
        mid = ch * ml + ((cl * ml) >> 16)
        mid2 = cl * mh + (mid & 0xFFFF)
        return ch * mh + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((cl * ml) & 0xFFFF)

    step = max(1, (1 << 24) // G)
    for t0 in range(0, T, step):
        n = min(step, T - t0)
        x = torch.empty(4, n, G, device="cuda", dtype=torch.int64)
        x[0] = torch.arange(G, device="cuda")
        x[1] = torch.arange(t0, t0 + n, device="cuda")[:, None]
        x[2], x[3] = s["offset"] % (1 << 32), s["offset"] // (1 << 32)
        for r in range(10):
            key = ((s["seed"] % (1 << 32) + r * 0x9E3779B9) % (1 << 32), (s["seed"] // (1 << 32) + r * 0xBB67AE85) % (1 << 32))
            (h0, l0), (h1, l1) = times(x[0], 0xD2511F53), times(x[2], 0xCD9E8D57)
            x = torch.stack([h1 ^ x[1] ^ key[0], l1, h0 ^ x[3] ^ key[1], l0])
        bits = torch.stack([x % 65536, x // 65536], -1)                    # [4, n, G, 2]
        keep[t0:t0 + n] = bits.permute(1, 2, 0, 3).reshape(n, G * 8) >= round(case["p"] * 65536)
    left = 1.0 - round(case["p"] * 65536) / 65536.0
    out = s["x"].to(d) / left * keep[:, :H]
    return out if s["residual"] is None else out + s["residual"].to(d)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("ffn", "ffn_bwd"):
        return _exact_ffn(s)
    if case["kind"] in ("scan", "scan_bwd"):
        return _exact_scan(s)
    return _exact_step(s) if case["kind"] == "scan_step" else _exact_dropout(s)
