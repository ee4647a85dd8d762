"""Residual norm, forward and backward, against the formulas in fp64.

Tolerances, before any run.  u is the output type's unit roundoff (bf16 2^-8, fp16
2^-11 and 2^-25 for its subnormals, fp32 2^-24).  Every output is a short chain of fp32
operations on sums over H, so it is off by at most GAMMA times the same formula with all
terms taken absolutely: a sum over H is at most 32 terms in a thread (loop kernels: H /
512 = 40 at the longest row here) and a tree of depth 14, around which each chain has at
most 20 operations, of which rsqrtf is 2 ulp: GAMMA = 96 * 2^-24.  Weights' gradients add
up to T more terms: (T + 96) 2^-24."""
import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}
GAMMA = 96 * 2.0**-24
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def dev():
    return torch.device("cuda", torch.cuda.current_device())


def make(T, H, dtype, res, ptype, post, gate, pre, residual, offset, seed=0, stride=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)

    def rows(scale, dt):
        v = (n(T, H) * scale).to(dev(), dt)
        if stride:
            wide = torch.full((T, H + stride), float("nan"), dtype=dt, device=dev())
            wide[:, :H] = v
            v = wide[:, :H]
        return v

    s = {"x": rows(1.0, dtype), "residual": rows(2.0, res) if residual else None, "eps": 1e-5, "alpha": 0.75,
         "offset": offset,
         "w_post": (1 - offset + 0.3 * n(H)).to(dev(), ptype) if post else None,
         "w_pre": (1 - offset + 0.3 * n(H)).to(dev(), ptype) if pre else None, "gate": None}
    if gate == "channel":
        s["gate"] = n(H).to(dev(), ptype)
    elif gate == "token":
        s["gate"] = n(T, 1).to(dev())
    elif gate == "full":
        s["gate"] = n(T, H).to(dev(), dtype)
    s["dy"] = rows(0.5, dtype) if pre else None
    s["dr"] = n(T, H).to(dev(), res)
    return s


def d64(t):
    return None if t is None else t.double()


def reference_fwd(s):
    """fp64 outputs, and the magnitudes that the error bound multiplies."""
    f = lambda v: float(np.float32(v))
    x, r, g = d64(s["x"]), d64(s["residual"]), d64(s["gate"])
    u, rstd_post = x, None
    if s["w_post"] is not None:
        rstd_post = 1 / torch.sqrt((x * x).mean(1) + f(s["eps"]))
        u = x * rstd_post[:, None] * (d64(s["w_post"]) + s["offset"])
        # (a weight near -offset cancels; the stored weight is exact, the sum is one rounding)
    if g is not None:
        u = u * g
    base = 0.0 if r is None else f(s["alpha"]) * r
    rp = base + u
    mag = (base.abs() if r is not None else 0.0) + u.abs()
    out = {"residual": (rp, mag), "rstd_post": None, "rstd_pre": None, "y": None}
    if rstd_post is not None:
        out["rstd_post"] = (rstd_post, rstd_post)
    if s["w_pre"] is not None:
        rstd = 1 / torch.sqrt((rp * rp).mean(1) + f(s["eps"]))
        # relative error of the mean of squares: twice that of r' in the 2-norm
        rel = (mag * mag).mean(1).sqrt() * rstd
        w = d64(s["w_pre"]) + s["offset"]
        out["rstd_pre"] = (rstd, rstd * (1 + 2 * rel))
        out["y"] = (rp * rstd[:, None] * w, (mag + rp.abs() * 2 * rel[:, None]) * rstd[:, None] * w.abs())
    return out


def reference_bwd(s, rp, rstd_post, rstd_pre):
    f = lambda v: float(np.float32(v))
    T, H = s["x"].shape
    zero = torch.zeros(T, H, dtype=torch.float64, device=dev())
    out = {"dw_pre": None, "dw_post": None, "dgate": None}
    t = zero if s["dr"] is None else d64(s["dr"])
    tm = t.abs()
    n = q = zero
    rstd = torch.zeros(T, 1, dtype=torch.float64, device=dev())
    if s["w_pre"] is not None:
        rstd = d64(rstd_pre)[:, None]
        n = d64(rp) * rstd
        q = d64(s["dy"]) * (d64(s["w_pre"]) + s["offset"])
        out["dw_pre"] = ((d64(s["dy"]) * n).sum(0), (d64(s["dy"]) * n).abs().sum(0))
    m_qn, m_qn_mag = (q * n).mean(1, keepdim=True), (q * n).abs().mean(1, keepdim=True)
    D = t + rstd * (q - n * m_qn)
    Dm = tm + rstd * (q.abs() + n.abs() * m_qn_mag)
    out["dresidual"] = (f(s["alpha"]) * D, f(s["alpha"]) * Dm)
    x, g = d64(s["x"]), d64(s["gate"])
    m = x if s["w_post"] is None else x * d64(rstd_post)[:, None]
    w = torch.ones(H, dtype=torch.float64, device=dev()) if s["w_post"] is None else d64(s["w_post"]) + s["offset"]
    du = D if g is None else D * g
    dum = Dm if g is None else Dm * g.abs()
    if g is not None:
        Du, Dum = D * (m * w), Dm * (m * w).abs()
        dim = {(H,): 0, (T, 1): 1}.get(tuple(g.shape))
        out["dgate"] = (Du, Dum) if dim is None else (Du.sum(dim), Dum.sum(dim))
    if s["w_post"] is None:
        out["dx"] = (du, dum)
        return out
    out["dw_post"] = ((du * m).sum(0), (dum * m.abs()).sum(0))
    p, pm = du * w, dum * w.abs()
    rs = d64(rstd_post)[:, None]
    out["dx"] = (rs * (p - m * (p * m).mean(1, keepdim=True)),
                 rs * (pm + m.abs() * (pm * m.abs()).mean(1, keepdim=True)))
    return out


def close(got, ref, gamma, name):
    if ref is None:
        assert got is None, name
        return
    v, mag = ref
    err = (got.double() - v).abs()
    lim = U[got.dtype] * v.abs() + gamma * mag + TINY[got.dtype]
    assert (err <= lim).all(), f"{name}: {float((err / lim.clamp_min(1e-300)).max()):.2f} of the bound"


def run_both(s, T):
    got = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"],
                                 res_scale=s["alpha"], eps=s["eps"], weight_offset=s["offset"])
    ref = reference_fwd(s)
    for k in ("y", "residual", "rstd_post", "rstd_pre"):
        close(got[k], ref[k], GAMMA, k)
    kw = dict(rstd_post=got["rstd_post"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], res_scale=s["alpha"],
              weight_offset=s["offset"], want_dresidual=True)
    back = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], got["residual"], got["rstd_pre"], **kw)
    rb = reference_bwd(s, got["residual"], got["rstd_post"], got["rstd_pre"])
    for k in ("dx", "dresidual"):
        close(back[k], rb[k], GAMMA, k)
    for k in ("dw_post", "dgate", "dw_pre"):
        close(back[k], rb[k], GAMMA + T * 2.0**-24, k)
    again = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], got["residual"], got["rstd_pre"], **kw)
    for k, v in back.items():
        assert v is None or torch.equal(v, again[k]), k
    return got, back


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre,residual", [(True, True, True), (False, True, True), (True, False, True),
                                               (False, True, False), (True, True, False)])
@pytest.mark.parametrize("T,H", [(1, 64), (5, 320), (37, 1031), (3, 4096)])
def test_parts(T, H, post, pre, residual, gate):
    run_both(make(T, H, BF, BF, F, post, gate, pre, residual, 0.0, seed=T + H), T)


@pytest.mark.parametrize("dtype,res,ptype", [(BF, F, BF), (HF, HF, F), (HF, F, HF), (F, F, F), (BF, BF, BF)])
@pytest.mark.parametrize("T,H", [(1, 1), (2, 3), (130, 8), (9, 255), (700, 256), (33, 264), (11, 5120), (3, 8192),
                                 (2, 8200), (2, 16384), (5, 5119), (2, 16383), (3, 20000), (2, 20001)])
def test_types_and_row_lengths(T, H, dtype, res, ptype):
    run_both(make(T, H, dtype, res, ptype, True, "channel", True, True, 1.0, seed=H), T)


@pytest.mark.parametrize("T,H", [(4000, 64), (3001, 320), (2500, 1000), (1500, 1001)])
def test_many_rows(T, H):
    run_both(make(T, H, BF, F, BF, True, "channel", True, True, 0.0, seed=1), T)


@pytest.mark.parametrize("dtype,res,ptype,gate", [(BF, F, BF, "channel"), (HF, HF, F, "full"), (F, F, F, "token"), (BF, BF, BF, "none")])
@pytest.mark.parametrize("T,H,stride", [(1, 2, 0), (900, 34, 0), (700, 250, 2), (5000, 1566, 0), (300, 514, 6), (40, 2050, 0),
                                        (9, 5122, 2), (7, 8190, 0), (3, 8198, 0), (3, 16386, 0)])
def test_rows_of_whole_pairs(T, H, stride, dtype, res, ptype, gate):
    """Even rows that are no multiple of eight, rows that begin at a pair but not at a vector."""
    run_both(make(T, H, dtype, res, ptype, True, gate, True, True, 0.0, seed=T + H, stride=stride), T)


@pytest.mark.parametrize("stride", [1, 8, 64])
@pytest.mark.parametrize("H", [64, 1024, 1025])
def test_strided_rows(H, stride):
    """Rows of a wider matrix, as a fused projection leaves them; what lies between them is NaN."""
    s = make(50, H, BF, BF, BF, True, "full", True, True, 0.0, seed=2, stride=stride)
    got, back = run_both(s, 50)
    whole = {k: v.contiguous() if torch.is_tensor(v) else v for k, v in s.items()}
    same, _ = run_both(whole, 50)
    if H % 8 == 0 and stride % 8 == 0:
        assert torch.equal(got["y"], same["y"]) and torch.equal(got["residual"], same["residual"])


def test_plain_norm_passes_the_stream_through():
    s = make(20, 256, BF, BF, BF, False, "none", True, False, 0.0)
    out = molt.residual_norm_fwd(s["x"], w_pre=s["w_pre"], eps=1e-5)
    assert out["residual"] is s["x"]
    x = s["x"].double()
    ref = x / torch.sqrt((x * x).mean(1, keepdim=True) + float(np.float32(1e-5))) * s["w_pre"].double()
    close(out["y"], (ref, ref.abs()), GAMMA, "y")
    wide = molt.residual_norm_fwd(s["x"], w_pre=s["w_pre"], residual_dtype=F)
    assert wide["residual"].dtype == F and torch.equal(wide["residual"], s["x"].float())


def test_serving_form_keeps_no_statistics():
    s = make(1, 4096, BF, BF, BF, True, "none", True, True, 0.0)
    out = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], w_pre=s["w_pre"], want_stats=False)
    full = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], w_pre=s["w_pre"])
    assert out["rstd_post"] is None and out["rstd_pre"] is None
    assert torch.equal(out["y"], full["y"]) and torch.equal(out["residual"], full["residual"])


def test_rows_do_not_touch_one_another():
    """A row of zeros, of the types' largest values, of NaN and of infinities."""
    s = make(40, 512, BF, F, F, True, "channel", True, True, 0.0, seed=3)
    ref = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    x, r = s["x"].clone(), s["residual"].clone()
    x[3], r[3] = 0.0, 0.0
    x[10, 5] = float("nan")
    r[20, 7] = float("inf")
    x[30] = 3e38
    out = molt.residual_norm_fwd(x, r, w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    assert (out["y"][3] == 0).all() and torch.isfinite(out["rstd_pre"][3])
    assert torch.isnan(out["y"][10]).all()
    assert torch.isnan(out["y"][20, 7]) and torch.isinf(out["residual"][20, 7])
    rest = [t for t in range(40) if t not in (3, 10, 20, 30)]
    assert torch.equal(out["y"][rest], ref["y"][rest]) and torch.equal(out["residual"][rest], ref["residual"][rest])


def test_accumulated_weight_gradients():
    s = make(300, 320, BF, BF, F, True, "channel", True, True, 0.0, seed=4)
    got, back = run_both(s, 300)
    bufs = {k: torch.randn(320, device=dev()) for k in ("dw_post", "dgate", "dw_pre")}
    before = {k: v.clone() for k, v in bufs.items()}
    molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], got["residual"], got["rstd_pre"], rstd_post=got["rstd_post"],
                           w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], res_scale=s["alpha"], accumulate=True,
                           **bufs)
    for k in bufs:
        assert torch.equal(bufs[k], before[k] + back[k]), k


def test_without_later_gradient():
    """The stream ends here: dresidual is None."""
    s = make(50, 640, BF, BF, BF, False, "none", True, True, 0.0, seed=5)
    s["dr"] = None
    run_both(s, 50)


def test_residual_in_place():
    s = make(33, 1031, BF, F, BF, True, "token", True, True, 0.0, seed=6)
    out = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    import ctypes
    from paper_2607_21653_gb300 import stream as S
    for H in (1031, 1024):
        x, r = s["x"][:, :H].contiguous(), s["residual"][:, :H].contiguous()
        wp, wq = s["w_post"][:H].contiguous(), s["w_pre"][:H].contiguous()
        out = molt.residual_norm_fwd(x, r, w_post=wp, gate=s["gate"], w_pre=wq)
        desc = S.NormDesc(33, H, 0, 0, 0, 0, 2, 0, S.GATE_TOKEN, 1.0, 1e-6, 0.0)
        y = torch.empty_like(x)
        st = molt.load().molt_residual_norm_fwd(ctypes.byref(desc), x.data_ptr(), r.data_ptr(), wp.data_ptr(),
                                                s["gate"].data_ptr(), wq.data_ptr(), y.data_ptr(), r.data_ptr(), None,
                                                None, torch.cuda.current_stream().cuda_stream)
        assert st == 0
        assert torch.equal(y, out["y"]) and torch.equal(r, out["residual"])


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_backward_by_differences(gate):
    """d/de of <y, dy> + <r', dr> along a random direction of every input, by central
    differences of the forward in fp32.  The step's own error is of third order (e = 2e-3)
    and fp32 rounding 2^-24 of the sums over e: 1e-3 of the sums covers both."""
    T, H = 24, 192
    s = make(T, H, F, F, F, True, gate, True, True, 0.0, seed=7)
    fwd = lambda s: molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"],
                                           res_scale=s["alpha"], eps=s["eps"])
    o = fwd(s)
    back = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], o["residual"], o["rstd_pre"], rstd_post=o["rstd_post"],
                                  w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"], res_scale=s["alpha"])
    value = lambda o: float((o["y"].double() * s["dy"].double()).sum() + (o["residual"].double() * s["dr"].double()).sum())
    size = float((o["y"].double() * s["dy"].double()).abs().sum() + (o["residual"].double() * s["dr"].double()).abs().sum())
    pairs = [("x", "dx"), ("residual", "dresidual"), ("w_post", "dw_post"), ("w_pre", "dw_pre")]
    if gate != "none":
        pairs.append(("gate", "dgate"))
    e = 2e-3
    for name, dname in pairs:
        step = torch.randn(s[name].shape, device=dev())
        plus, minus = dict(s), dict(s)
        plus[name], minus[name] = s[name] + e * step, s[name] - e * step
        got = (value(fwd(plus)) - value(fwd(minus))) / (2 * e)
        want = float((back[dname].double().reshape(step.shape) * step.double()).sum())
        assert abs(got - want) <= 1e-3 * size, (name, got, want)


def test_no_rows():
    s = make(0, 64, BF, BF, BF, True, "channel", True, True, 0.0)
    out = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    assert out["y"].shape == (0, 64)
    back = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], out["residual"], out["rstd_pre"],
                                  rstd_post=out["rstd_post"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    assert all((back[k] == 0).all() for k in ("dw_post", "dw_pre", "dgate"))


def test_other_stream_and_workspace():
    s = make(500, 768, BF, BF, BF, True, "channel", True, True, 0.0, seed=8)
    o = molt.residual_norm_fwd(s["x"], s["residual"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    kw = dict(rstd_post=o["rstd_post"], w_post=s["w_post"], gate=s["gate"], w_pre=s["w_pre"])
    ref = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], o["residual"], o["rstd_pre"], **kw)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], o["residual"], o["rstd_pre"], **kw)
    torch.cuda.current_stream().wait_stream(st)
    for k, v in ref.items():
        assert torch.equal(v, got[k]), k
    with pytest.raises(molt.MoltError) as e:
        molt.residual_norm_bwd(s["dy"], s["dr"], s["x"], o["residual"], o["rstd_pre"],
                               workspace=torch.empty(300, dtype=torch.uint8, device=dev()), **kw)
    assert e.value.status == 9
