"""Gates far below 0 in the recurrence: what is left of a large state (or of a large gradient) behind one is a
multiple of a small a = e^gate or so, and is held against that, not against the state.

Tolerances, before any run.  e^gate is off by |gate| 2^-23 of itself for its argument gate log2 e
(the constant's and the product's rounding, 2^-24 each) and by 2^-22 for the function; a sum with 1,
a reciprocal and a product add 2^-22 to a, and as much to 1 - a:
  d = |gate| 2^-23 + 2^-21.
Of 16-bit inputs with gates not below -4.875 a is 1 + (a - 1) in fp32: 2^-22 of 1 more, 2^-22 / a of it.
What enters a row has the size S, the sum of the absolute values in it:
  S_t = a S_{t-1} + (1 - a) |v|,   err_t = a err_{t-1} + 4 (d a S_{t-1} + d (1 - a) |v| + 2^-23 S_t)
(four times: rows' maps are composed over warps and tiles besides), log form with |v| for
(1 - a) |v|; the same for E from the other end with dy, and products by their factors' errors.
Results below 2^-120 may be lost, and those of fp16 past 65504 are infinite, as any rounding to
fp16 makes them (dgate here, of states and gradients of 1000); results in 16 bits are off by a rounding more (bf16 2^-8, fp16
2^-11, and half the smallest subnormal, 2^-25)."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 0.0}
TINY = {torch.bfloat16: 2.0**-120, torch.float16: 2.0**-25, torch.float32: 2.0**-120}
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
GATES = (-2.0, -4.0, -4.75, -4.875, -5.0, -6.0, -8.0, -10.0, -12.0, -14.0, -16.0, -18.0, -20.0)
TIMES = 4.0


def parts(f, kind, dtype):
    """a, what v is multiplied by, and a's relative error."""
    a = torch.sigmoid(f) if kind == "sigmoid" else torch.exp(f)
    w = torch.sigmoid(-f) if kind == "sigmoid" else torch.ones_like(f)
    d = f.abs() * 2.0**-23 + 2.0**-21
    return a, w, d, d if dtype == torch.float32 else torch.where(f < -4.875, d, d + 2.0**-22 / a)


def reference(s, cu, kind):
    dtype = s["gate"].dtype
    f, v, dy = (s[k].double() for k in ("gate", "value", "dy"))
    T, H = f.shape
    a, w, d, da = parts(f, kind, dtype)
    z = lambda *n: torch.zeros(*n, device=f.device, dtype=torch.float64)
    B = len(cu) - 1
    h, eh, hp, ehp, shp, D, eD, E, eE, sE = (z(T, H) for _ in range(10))
    fin, efin, ini, eini = z(B, H), z(B, H), z(B, H), z(B, H)
    for b in range(B):
        at, e, S = s["h0"][b].double(), z(H), s["h0"][b].double().abs()
        for t in range(cu[b], cu[b + 1]):
            hp[t], ehp[t], shp[t] = at, e, S
            new_S = a[t] * S + w[t] * v[t].abs()
            e = a[t] * e + TIMES * (da[t] * a[t] * S + d[t] * w[t] * v[t].abs() + 2.0**-23 * new_S)
            at, S = a[t] * at + w[t] * v[t], new_S
            h[t], eh[t] = at, e
        fin[b], efin[b] = at, e
        at, e = s["dfinal"][b].double(), z(H)
        S = at.abs()
        for t in range(cu[b + 1] - 1, cu[b] - 1, -1):
            D[t], S = dy[t] + at, dy[t].abs() + S
            eD[t] = e + TIMES * 2.0**-23 * S
            at, S = a[t] * D[t], a[t] * S
            e = a[t] * eD[t] + TIMES * (da[t] * S + 2.0**-23 * S)
            E[t], eE[t], sE[t] = at, e, S
        ini[b], eini[b] = at, e
    wE = w if kind == "sigmoid" else torch.ones_like(w)
    x, sx = (hp - v, shp + v.abs()) if kind == "sigmoid" else (hp, shp)
    dg = E * wE * x
    edg = wE * (eE * x.abs() + (E.abs() + eE) * ehp) + (d + 2.0**-21) * wE * (E.abs() + eE) * sx
    return {"y": (h, eh), "final_state": (fin, efin), "dinitial_state": (ini, eini), "dgate": (dg, edg),
            "dvalue": (D * wE, wE * eD + (d + 2.0**-22) * wE * D.abs())}


def check(got, ref, what):
    r, e = ref
    bound = e + U[got.dtype] * (r.abs() + e) + TINY[got.dtype]
    # what is rounded past the type's largest value is infinite; next to it either is right
    most = torch.finfo(got.dtype).max
    over = r.abs() - e > most * (1 + 2.0**-8)
    assert (got[over].double() == r[over].sign() * float("inf")).all(), what
    err = torch.where(over | (got.isinf() & (r.abs() + bound > most)), 0.0, (got.double() - r).abs())
    assert (err <= bound).all(), (what, float((err / bound).max()), float((err / (r.abs() + 1e-300))[err > bound].max()))


def run(s, cu, kind):
    c = torch.tensor(cu, dtype=torch.int32, device=dev())
    out = molt.gated_scan_fwd(s["gate"], s["value"], initial_state=s["h0"], cu_seqlens=c, kind=kind, want_states=True)
    out.update(molt.gated_scan_bwd(s["dy"], s["gate"], s["value"], out["states"], initial_state=s["h0"], cu_seqlens=c,
                                   dfinal_state=s["dfinal"], kind=kind))
    return out


def everything(s, cu, kind):
    ref, out = reference(s, cu, kind), run(s, cu, kind)
    for k, r in ref.items():
        check(out[k], r, k)


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,aligned", [(13 * 16, True), (13 * 5, False)])
def test_nothing_but_what_is_left_of_a_state(H, aligned, dtype, kind):
    """Values of 0 (and no gradient but the final state's and the last row's): h and E are products of a alone."""
    g = torch.Generator(device=dev()).manual_seed(1)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    for cu in ([0, 1], [0, 3], [0, 1, 3, 6, 7, 9, 11, 12, 14, 17], [0, 2, 20, 23, 130, 132]):
        T, B = cu[-1], len(cu) - 1
        s = {"gate": torch.tensor(GATES, device=dev()).repeat(H // 13).expand(T, H).contiguous().to(dtype),
             "value": torch.zeros(T, H, dtype=dtype, device=dev()), "dy": torch.zeros(T, H, dtype=dtype, device=dev()),
             "h0": n(B, H), "dfinal": n(B, H)}
        if T > 20:   # one long sequence whose rows but a few remember all
            s["gate"][2:20, ::2] = 5.0 if kind == "sigmoid" else -0.01
            s["gate"][23:128] = 5.0 if kind == "sigmoid" else -0.01
        s["dy"][-1] = n(H).to(dtype)
        everything(s, cu, kind)


def resets(T, H, B, dtype, kind):
    """Small values, and large ones that the next row's gate takes back; dy the other way round."""
    g = torch.Generator(device=dev()).manual_seed(2)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    gate = torch.full((T, H), 3.0 if kind == "sigmoid" else -0.05, device=dev())
    value, dy = 1e-3 * n(T, H), 1e-3 * n(T, H)
    low = torch.tensor(GATES, device=dev()).repeat(H // 13)
    for t in range(3, T, 9):
        gate[t] = low.roll(t)
        value[t - 1], dy[t] = 1000.0, 1000.0
    return {"gate": gate.to(dtype), "value": value.to(dtype), "dy": dy.to(dtype), "h0": n(B, H), "dfinal": n(B, H)}


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cu", [[0, 300], [0, 7, 150, 151, 300], list(range(0, 301, 20))])
@pytest.mark.parametrize("H", [13 * 8, 13 * 7])
def test_resets_of_large_states(H, cu, dtype, kind):
    everything(resets(300, H, len(cu) - 1, dtype, kind), cu, kind)


@pytest.mark.parametrize("dtype,kind,H", [(torch.bfloat16, "sigmoid", 13 * 8), (torch.float16, "log", 13 * 5), (torch.float32, "sigmoid", 13 * 4)])
def test_resets_in_segments(dtype, kind, H):
    """Rows enough for segments, whose maps are formed by a launch of their own."""
    cu = [0, 9000, 18000]
    everything(resets(18000, H, 2, dtype, kind), cu, kind)


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H", [13 * 4, 13])
def test_step(H, dtype, kind):
    g = torch.Generator(device=dev()).manual_seed(3)
    for scale in (0.0, 1e-3):
        gate = torch.tensor(GATES, device=dev()).repeat(H // 13).expand(5, H).contiguous().to(dtype)
        value = (scale * torch.randn(5, H, device=dev(), generator=g)).to(dtype)
        state = 1000 * torch.randn(5, H, device=dev(), generator=g)
        out = molt.gated_scan_step(gate, value, state, kind=kind)
        a, w, d, _ = parts(gate.double(), kind, torch.float32)
        h, v = state.double(), value.double()
        ref = a * h + w * v
        e = TIMES * (d * a * h.abs() + d * w * v.abs() + 2.0**-23 * (a * h.abs() + w * v.abs()))
        check(out["state"], (ref, e), "state")
        check(out["y"], (ref, e), "y")
