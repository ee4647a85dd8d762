"""Gated feed-forward block and its gradients, against fp64 on the device.

Tolerances, before any run, element by element.  u is half a step of the 16-bit type
(bf16 2^-8, fp16 2^-11), t half its smallest subnormal (fp16 2^-25).
  a sum of K products on the tensor cores: (K / 8 + 8) 2^-23 of the sum of their absolute
    values (fp32, bits below a block's largest term cut off; K / 16 blocks);
  act and act' in fp32: e^x with |x| up to 300 is off by 2^-22 + |x| 2^-23 of itself where
    the argument is rounded, which counts where the result is not yet 0 or 1, |x| < 20: 2^-17
    of act, and 2^-17 * 1.5 for act' (|act'| < 1.13, |act''| < 0.8);
  a rounding: u of the value, plus t.
They are carried through the formulas by absolute values: a bound for any signs of the
roundings.  They are independent, so for a whole tensor of 4096 elements or more
the norm of the error is within 2 u of the norm of the result: u for the last
rounding, and u for those before it (u / sqrt 3 each, at most three in a sum).  Two
more u where g and u are rounded themselves before they are used does not occur: they are
inputs of the backward, or formed again in fp32."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 0.0}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
ACT_REL = 2.0**-17


def act64(name, g):
    """act(g), act'(g) from autograd."""
    F = torch.nn.functional
    f = {"silu": F.silu, "relu": F.relu, "gelu": lambda t: F.gelu(t, approximate="tanh")}[name]
    g = g.detach().requires_grad_(True)
    a = f(g)
    d, = torch.autograd.grad(a.sum(), g)
    return a.detach(), d


def acc(K):
    return (K / 8 + 8) * 2.0**-23


def inputs(T, H, F, dtype, seed, scale=1.0):
    g = torch.Generator(device=dev()).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    return {"x": n(T, H).to(dtype), "w_gate": (n(F, H) * H**-0.5 * scale).to(dtype), "w_up": (n(F, H) * H**-0.5).to(dtype),
            "w_down": (n(H, F) * F**-0.5).to(dtype), "dy": (0.1 * n(T, H)).to(dtype)}


def product(a, b, ea=None, eb=None):
    """a @ b.t(), and the bound for its error where a and b are off by ea and eb."""
    K = a.shape[1]
    c = a @ b.t()
    e = acc(K) * (a.abs() @ b.abs().t())
    if ea is not None:
        e = e + ea @ (b.abs() + (0 if eb is None else eb)).t()
    if eb is not None:
        e = e + a.abs() @ eb.t()
    return c, e


def rounded(v, e, dtype):
    return e + U[dtype] * (v.abs() + e) + TINY[dtype]


def check(got, ref, bound, dtype, what):
    assert got.dtype == dtype and got.shape == ref.shape, what
    err = (got.double() - ref).abs()
    worst = (err - bound).max()
    assert (err <= bound).all(), (what, float(worst), float(err.max()))
    if ref.numel() >= 4096:
        u = max(U[dtype], 0.0)
        assert float(err.norm()) <= (2 * u if u else 1.0) * float(ref.norm()), what


def fwd_reference(s, act, dtype):
    d = {k: v.double() for k, v in s.items()}
    g, eg = product(d["x"], d["w_gate"])
    u, eu = product(d["x"], d["w_up"])
    a, _ = act64(act, g)
    ea = 1.13 * eg + ACT_REL * a.abs()
    h = a * u
    eh = rounded(h, ea * (u.abs() + eu) + a.abs() * eu + 2.0**-23 * h.abs(), dtype)
    y, ey = product(h, d["w_down"], eh)
    return {"gate": (g, rounded(g, eg, dtype)), "up": (u, rounded(u, eu, dtype)), "y": (y, rounded(y, ey, dtype))}


SHAPES = [(1, 8, 8), (1, 64, 64), (2, 4096, 72), (3, 72, 200), (8, 640, 2392), (9, 512, 1000), (33, 1024, 264), (130, 64, 136),
          (257, 328, 264), (300, 896, 2392), (512, 2048, 5504), (1031, 896, 2392), (5000, 64, 64), (700, 2040, 8)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("T,H,F", SHAPES)
def test_forward(T, H, F, dtype):
    s = inputs(T, H, F, dtype, T + H)
    for act in ("silu", "gelu", "relu"):
        ref = fwd_reference(s, act, dtype)
        w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
        out = molt.gated_ffn_fwd(*w, activation=act, keep=True)
        for k, (r, b) in ref.items():
            check(out[k], r, b, dtype, (act, k))
        plain = molt.gated_ffn_fwd(*w, activation=act)
        assert plain["gate"] is None and plain["up"] is None
        assert torch.equal(plain["y"], out["y"])
    assert molt.device_status() == 0


def bwd_reference(s, act, dtype, gate=None, up=None):
    d = {k: v.double() for k, v in s.items()}
    if gate is None:
        g, eg = product(d["x"], d["w_gate"])
        u, eu = product(d["x"], d["w_up"])
    else:
        g, u = gate.double(), up.double()
        eg = eu = torch.zeros_like(g)
    a, da = act64(act, g)
    dh, edh = product(d["dy"], d["w_down"].t().contiguous())
    ea = 1.13 * eg + ACT_REL * a.abs()
    eda = 0.8 * eg + 1.5 * ACT_REL * torch.ones_like(g)
    if act == "relu":
        eda = (g.abs() <= eg).double()     # which branch is open there
    dg, du, h = dh * u * da, dh * a, a * u
    edg = edh * (u.abs() + eu) * (da.abs() + eda) + dh.abs() * (eu * (da.abs() + eda) + u.abs() * eda) + 2.0**-22 * dg.abs()
    edu = edh * (a.abs() + ea) + dh.abs() * ea + 2.0**-23 * du.abs()
    eh = ea * (u.abs() + eu) + a.abs() * eu + 2.0**-23 * h.abs()
    edg, edu, eh = rounded(dg, edg, dtype), rounded(du, edu, dtype), rounded(h, eh, dtype)
    t = lambda m: m.t().contiguous()
    both, eboth = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    w = torch.cat([d["w_gate"], d["w_up"]], 0)
    return {"dx": product(both, t(w), eboth), "dw_gate": product(t(dg), t(d["x"]), t(edg)),
            "dw_up": product(t(du), t(d["x"]), t(edu)), "dw_down": product(t(d["dy"]), t(h), None, t(eh))}


@pytest.mark.parametrize("dtype,dw_dtype", [(BF, BF), (BF, F32), (HF, HF), (HF, F32)])
@pytest.mark.parametrize("T,H,F", SHAPES)
def test_gradients(T, H, F, dtype, dw_dtype):
    s = inputs(T, H, F, dtype, T + F)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
    for act, kept in (("silu", True), ("silu", False), ("gelu", False), ("relu", True)):
        k = molt.gated_ffn_fwd(*w, activation=act, keep=True) if kept else {"gate": None, "up": None}
        out = molt.gated_ffn_bwd(s["dy"], *w, gate=k["gate"], up=k["up"], activation=act, dw_dtype=dw_dtype)
        again = molt.gated_ffn_bwd(s["dy"], *w, gate=k["gate"], up=k["up"], activation=act, dw_dtype=dw_dtype)
        ref = bwd_reference(s, act, dtype, k["gate"], k["up"])
        for name, (r, e) in ref.items():
            to = dtype if name == "dx" else dw_dtype
            if to is F32:
                check(out[name], r, e + 2.0**-24 * r.abs(), F32, (act, kept, name))
                if r.numel() >= 4096:
                    assert float((out[name].double() - r).norm()) <= U[dtype] * float(r.norm()), (act, kept, name)
            else:
                check(out[name], r, rounded(r, e, to), to, (act, kept, name))
            assert torch.equal(out[name], again[name]), (act, kept, name)
    assert molt.device_status() == 0


@pytest.mark.parametrize("kept", [True, False])
def test_gradients_against_differences(kept):
    """d loss / d input along a direction, loss = sum y c, from the forward's own fp64 formula."""
    T, H, F, dtype = 37, 64, 128, HF
    s = inputs(T, H, F, dtype, 5)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
    k = molt.gated_ffn_fwd(*w, keep=True) if kept else {"gate": None, "up": None}
    out = molt.gated_ffn_bwd(s["dy"], *w, gate=k["gate"], up=k["up"])

    def loss(m):
        h = torch.nn.functional.silu(m["x"] @ m["w_gate"].t()) * (m["x"] @ m["w_up"].t())
        return float(((h @ m["w_down"].t()) * s["dy"].double()).sum())

    gen = torch.Generator(device=dev()).manual_seed(1)
    d = {n: v.double() for n, v in s.items()}
    for name, grad in (("x", out["dx"]), ("w_gate", out["dw_gate"]), ("w_up", out["dw_up"]), ("w_down", out["dw_down"])):
        v = torch.randn(d[name].shape, device=dev(), generator=gen, dtype=torch.float64)
        eps = 1e-5
        diff = (loss({**d, name: d[name] + eps * v}) - loss({**d, name: d[name] - eps * v})) / (2 * eps)
        got = float((grad.double() * v).sum())
        # each entry's error is within 4 u of its terms (two kept values, dg or du, the result); added with
        # independent signs, of grad's norm
        assert abs(got - diff) <= 4 * U[dtype] * float(grad.double().norm()) * 4, name


def test_strided_rows_and_slices():
    """Operands that are parts of larger tensors: a fused projection's halves, columns of a buffer."""
    T, H, F = 131, 136, 200
    s = inputs(T, H, F, BF, 3)
    wide = lambda t, extra: torch.cat([t, torch.full((t.shape[0], extra), 7.0, dtype=t.dtype, device=t.device)], 1)[:, :t.shape[1]]
    both = torch.cat([s["w_gate"], s["w_up"]], 0)
    want = molt.gated_ffn_fwd(s["x"], s["w_gate"], s["w_up"], s["w_down"], keep=True)
    x, wd, dy = wide(s["x"], 24), wide(s["w_down"], 8), wide(s["dy"], 64)
    got = molt.gated_ffn_fwd(x, both[:F], wide(both, 8)[F:], wd, keep=True)
    for k in want:
        assert torch.equal(want[k], got[k])
    a = molt.gated_ffn_bwd(s["dy"], s["x"], s["w_gate"], s["w_up"], s["w_down"])
    b = molt.gated_ffn_bwd(dy, x, both[:F], wide(both, 8)[F:], wd)
    for k in a:
        assert torch.equal(a[k], b[k])
    with pytest.raises(molt.MoltError, match="aligned|multiples"):
        molt.gated_ffn_fwd(wide(s["x"], 4), s["w_gate"], s["w_up"], s["w_down"])
    with pytest.raises(ValueError, match="contiguous rows"):
        molt.gated_ffn_fwd(s["x"], s["w_gate"].t().contiguous().t(), s["w_up"], s["w_down"])


def test_accumulate_and_given_buffers():
    T, H, F = 200, 64, 128
    s = inputs(T, H, F, BF, 4)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
    one = molt.gated_ffn_bwd(s["dy"], *w)
    bufs = {n: torch.full_like(one[n], 3.0) for n in ("dw_gate", "dw_up", "dw_down")}
    out = molt.gated_ffn_bwd(s["dy"], *w, accumulate=True, **bufs)
    for n, t in bufs.items():
        assert out[n] is t
        # one addition in fp32
        assert ((t.double() - (3.0 + one[n].double())).abs() <= 2.0**-24 * t.double().abs()).all(), n
    out = molt.gated_ffn_bwd(s["dy"], *w, **bufs)
    for n in bufs:
        assert torch.equal(out[n], one[n])
    with pytest.raises(ValueError, match="all three"):
        molt.gated_ffn_bwd(s["dy"], *w, dw_gate=bufs["dw_gate"])
    with pytest.raises(molt.MoltError, match="fp32 only"):
        molt.gated_ffn_bwd(s["dy"], *w, dw_dtype=BF, accumulate=True)
    with pytest.raises(ValueError, match="together"):
        molt.gated_ffn_bwd(s["dy"], *w, gate=torch.zeros(T, F, dtype=BF, device=dev()))


def test_no_tokens():
    s = inputs(0, 64, 128, BF, 4)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
    out = molt.gated_ffn_fwd(*w, keep=True)
    assert out["y"].shape == (0, 64) and out["gate"].shape == (0, 128)
    g = molt.gated_ffn_bwd(s["dy"], *w)
    assert all((g[n] == 0).all() for n in ("dw_gate", "dw_up", "dw_down"))
    kept = {n: torch.full_like(g[n], 2.0) for n in ("dw_gate", "dw_up", "dw_down")}
    molt.gated_ffn_bwd(s["dy"], *w, accumulate=True, **kept)
    assert all((t == 2).all() for t in kept.values())


def test_a_row_stays_its_own():
    """An infinity and a NaN in one token reach no other, and rows past the end take no part."""
    T, H, F = 70, 64, 128
    s = inputs(T, H, F, BF, 9)
    w = (s["w_gate"], s["w_up"], s["w_down"])
    want = molt.gated_ffn_fwd(s["x"], *w)["y"]
    x = s["x"].clone()
    x[3, 5], x[11, 0] = float("inf"), float("nan")
    got = molt.gated_ffn_fwd(x, *w)["y"]
    rest = [i for i in range(T) if i not in (3, 11)]
    assert torch.equal(got[rest], want[rest]) and got[11].isnan().all()


def test_two_streams_at_once():
    """Calls on two streams have workspaces of their own."""
    s = [inputs(600, 512, 1024, BF, i) for i in (1, 2)]
    args = lambda m: (m["x"], m["w_gate"], m["w_up"], m["w_down"])
    want = [molt.gated_ffn_bwd(m["dy"], *args(m)) for m in s]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in s]
    got = [None, None]
    for _ in range(4):
        for i, m in enumerate(s):
            with torch.cuda.stream(streams[i]):
                got[i] = molt.gated_ffn_bwd(m["dy"], *args(m))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for k in a:
            assert torch.equal(a[k], b[k])


def test_calls_one_after_another_without_a_wait():
    """Launches begin while the ones before them end: calls of many sizes on one workspace, each
    input the output of the call before, have the bits that they have one by one."""
    H, F, sizes = 256, 704, (1, 16, 17, 300, 5, 1031, 2, 600, 1)
    s = inputs(1031, H, F, BF, 3)
    w = (s["w_gate"], s["w_up"], s["w_down"])

    def calls(wait):
        x, out = s["x"], []
        for T in sizes * 4:
            f = molt.gated_ffn_fwd(x[:T], *w, keep=True)
            g = molt.gated_ffn_bwd(x[:T], f["y"], *w, *((f["gate"], f["up"]) if T % 2 else ()))
            x = x.clone()
            x[:T] = 0.5 * f["y"] + g["dx"] / (1 + g["dx"].abs().max())
            out += [f["y"], f["gate"], g["dx"], g["dw_gate"], g["dw_down"]]
            if wait:
                torch.cuda.synchronize()
        return out

    want = calls(True)
    for _ in range(3):
        for a, b in zip(want, calls(False)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 40, 600])
def test_in_two_captured_graphs(T):
    """Replayed in turn on new inputs, with the bits of the calls outside of them."""
    H, F = 256, 384
    s = inputs(T, H, F, BF, 6)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])

    def calls():
        out = molt.gated_ffn_fwd(*w, keep=True)
        return {**out, **molt.gated_ffn_bwd(s["dy"], *w, gate=out["gate"], up=out["up"])}

    calls()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(calls())
    for seed in (10, 11):
        new = inputs(T, H, F, BF, seed)
        s["x"].copy_(new["x"])
        s["dy"].copy_(new["dy"])
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = calls()
        for out in outs:
            for k in want:
                assert torch.equal(out[k], want[k]), k


def test_workspace_of_the_largest_batch_serves_smaller_ones():
    H, F = 256, 1000
    from paper_2607_21653_gb300 import blocks as B
    d = B.FfnDesc(2000, H, F, 0, 0, 0, 0, 0, 0, 0)
    lib = molt.load()
    ws = torch.empty(max(lib.molt_gated_ffn_fwd_workspace_bytes(ctypes.byref(d)),
                         lib.molt_gated_ffn_bwd_workspace_bytes(ctypes.byref(d), 0)), dtype=torch.uint8, device=dev())
    for T in (2000, 1999, 700, 257, 256, 129, 17, 8, 3, 1):
        s = inputs(T, H, F, BF, T)
        w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
        ws.fill_(255)      # NaN, wherever something is read that was not written
        a, b = molt.gated_ffn_fwd(*w, workspace=ws), molt.gated_ffn_fwd(*w)
        assert torch.equal(a["y"], b["y"])
        ws.fill_(255)
        a, b = molt.gated_ffn_bwd(s["dy"], *w, workspace=ws), molt.gated_ffn_bwd(s["dy"], *w)
        for k in a:
            assert torch.equal(a[k], b[k]), (T, k)
