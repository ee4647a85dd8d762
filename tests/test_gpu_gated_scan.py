"""Gated linear recurrence, its gradients and its step, against fp64 row by row on the device.

Tolerances, before any run, carried along the recurrence by absolute values.  1 - a in fp32 is
off by 2^-19 of itself for |gate| <= 20 (the exponential's argument is rounded: 20 log2 e
2^-24 ln 2 of e, and 2^-22 for the functions), so by n (2^-19); a step's own operations by
2^-23 of the values that enter; maps composed over a tile's warps repeat both, so four times
the sum of the two is allowed:
  err_t <= a err_{t-1} + 4 (2^-19 (1 - a) (|h| + |v|) + 2^-23 (|h_t| + |h_{t-1}| + |v|))
and the same for E, with D in the place of h.  Results in 16 bits: u of the value more (bf16
2^-8, fp16 2^-11 and half its smallest subnormal)."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}
TINY = {torch.bfloat16: 0.0, torch.float16: 2.0**-25, torch.float32: 0.0}
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
E_NA, E_OP, TIMES = 2.0**-19, 2.0**-23, 4.0
INF = float("inf")


def make(T, H, B, dtype, kind, seed, long=2.0):
    g = torch.Generator(device=dev()).manual_seed(seed)
    n = lambda *s: torch.randn(*s, device=dev(), generator=g)
    f = n(T, H) + long * 2 * torch.rand(H, device=dev(), generator=g)
    if kind == "log":
        f = -torch.log1p(torch.exp(-f))
    return {"gate": f.to(dtype), "value": n(T, H).to(dtype), "dy": n(T, H).to(dtype), "h0": n(B, H), "dfinal": n(B, H)}


def reference(s, cu, kind, with_state=True, grads=True):
    """Outputs in fp64 and the bounds of their errors in fp32, by name."""
    f, v, dy = (s[k].double() for k in ("gate", "value", "dy"))
    T, H = f.shape
    B = len(cu) - 1
    a = torch.sigmoid(f) if kind == "sigmoid" else torch.exp(f)
    na = torch.sigmoid(-f) if kind == "sigmoid" else -torch.expm1(f)
    z = lambda *shape: torch.zeros(*shape, device=f.device, dtype=torch.float64)
    h0 = s["h0"].double() if with_state else z(B, H)
    df = s["dfinal"].double() if with_state else z(B, H)
    h, eh, hp, ehp, D, eD = (z(T, H) for _ in range(6))
    fin, efin, ini, eini = h0.clone(), z(B, H), df.clone(), z(B, H)
    for b in range(B):
        at, e = h0[b], z(H)
        for t in range(cu[b], cu[b + 1]):
            hp[t], ehp[t] = at, e
            new = a[t] * at + (na[t] * v[t] if kind == "sigmoid" else v[t])
            e = a[t] * e + TIMES * (E_NA * na[t].abs() * (at.abs() + v[t].abs()) + E_OP * (new.abs() + at.abs() + v[t].abs()))
            at = new
            h[t], eh[t] = at, e
        fin[b], efin[b] = at, e
        at, e = df[b], z(H)
        for t in range(cu[b + 1] - 1, cu[b] - 1, -1):
            D[t], eD[t] = dy[t] + at, e + TIMES * E_OP * (dy[t].abs() + at.abs())
            at = a[t] * D[t]
            e = a[t] * eD[t] + TIMES * (E_NA * na[t].abs() * D[t].abs() + E_OP * D[t].abs())
        ini[b], eini[b] = at, e
    out = {"y": (h, eh), "final_state": (fin, efin), "dinitial_state": (ini, eini)}
    if kind == "sigmoid":
        w = a * na
        out["dvalue"] = D * na, eD * na + 4 * E_NA * (D * na).abs()
        x = hp - v
        out["dgate"] = D * x * w, eD * (x * w).abs() + ehp * (D * w).abs() + 8 * E_NA * (D * w).abs() * (hp.abs() + v.abs())
    else:
        out["dvalue"] = D, eD
        out["dgate"] = D * hp * a, eD * (hp * a).abs() + ehp * (D * a).abs() + 8 * E_NA * (D * hp).abs() * (a + na.abs())
    states = z((T + 127) // 128, H)
    es = z((T + 127) // 128, H)
    for k in range(1, states.shape[0]):
        states[k], es[k] = h[128 * k - 1], eh[128 * k - 1]
    out["states"] = states, es
    return out


def check(got, ref, dtype, what, rows=slice(None)):
    r, e = ref
    r, e = r[rows], e[rows]
    bound = e + U[dtype] * (r.abs() + e) + TINY[dtype]
    err = (got[rows].double() - r).abs()
    assert got.dtype == dtype and (err <= bound).all(), (what, float((err - bound).max()), float(err.max()))


def run(s, cu, kind, with_state=True, packed=True):
    c = torch.tensor(cu, dtype=torch.int32, device=dev()) if packed else None
    h0 = s["h0"] if with_state else None
    out = molt.gated_scan_fwd(s["gate"], s["value"], initial_state=h0, cu_seqlens=c, kind=kind, want_states=True)
    out.update(molt.gated_scan_bwd(s["dy"], s["gate"], s["value"], out["states"], initial_state=h0, cu_seqlens=c,
                                   dfinal_state=s["dfinal"] if with_state else None, kind=kind))
    return out


CUTS = {  # sequences over T rows, from none empty to most
    "one": lambda T: [0, T],
    "few": lambda T: sorted({0, T // 3, T // 2, T}),
    "empty": lambda T: [0, 0, T // 4, T // 4, T // 4, T - T // 5, T, T],
    "ones": lambda T: list(range(T + 1)),
    "inside": lambda T: [T // 5, T // 2, T // 2, T - T // 4],
}


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H", [(1, 1), (1, 64), (2, 130), (15, 63), (16, 64), (17, 66), (127, 8), (128, 65), (129, 320),
                                 (300, 96), (1031, 72)])
def test_against_rows(T, H, dtype, kind):
    for name, cut in CUTS.items():
        if name == "ones" and T > 300:
            continue
        cu = cut(T)
        B = len(cu) - 1
        s = make(T, H, B, dtype, kind, T + H)
        for with_state in (True, False):
            ref = reference(s, cu, kind, with_state)
            out = run(s, cu, kind, with_state)
            rows = slice(cu[0], cu[-1])
            for k in ("y", "dgate", "dvalue"):
                check(out[k], ref[k], dtype, (name, k), rows)
                assert (out[k][:cu[0]] == 0).all() and (out[k][cu[-1]:] == 0).all(), (name, k)
            check(out["final_state"], ref["final_state"], torch.float32, (name, "final"))
            if with_state:
                check(out["dinitial_state"], ref["dinitial_state"], torch.float32, (name, "dinitial"))
            if name != "inside":
                check(out["states"], ref["states"], torch.float32, (name, "states"))
            again = run(s, cu, kind, with_state)
            for k, v in out.items():
                assert v is None or torch.equal(v, again[k]), (name, k)
    assert molt.device_status() == 0


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_memory(dtype, kind):
    """Thousands of rows whose channels remember all of them, across many tiles."""
    T, H = 5003, 136
    s = make(T, H, 3, dtype, kind, 1, long=4.0)
    cu = [0, 4500, 4501, T]
    ref, out = reference(s, cu, kind), run(s, cu, kind)
    for k in ("y", "dgate", "dvalue"):
        check(out[k], ref[k], dtype, k)
    for k in ("final_state", "dinitial_state", "states"):
        check(out[k], ref[k], torch.float32, k)


@pytest.mark.parametrize("dtype,H", [(torch.bfloat16, 72), (torch.bfloat16, 65), (torch.float32, 40), (torch.float16, 33)])
def test_long_and_narrow(dtype, H):
    """Few channels and many rows: segments of rows, each of them several tiles to a block."""
    T = 18000
    s = make(T, H, 5, dtype, "sigmoid", 2, long=3.0)
    cu = [100, 100, 2500, 2600, 17000, T - 50]
    ref, out = reference(s, cu, "sigmoid"), run(s, cu, "sigmoid")
    rows = slice(cu[0], cu[-1])
    for k in ("y", "dgate", "dvalue"):
        check(out[k], ref[k], dtype, k, rows)
    for k in ("final_state", "dinitial_state"):
        check(out[k], ref[k], torch.float32, k)
    again = run(s, cu, "sigmoid")
    for k, v in out.items():
        assert torch.equal(v, again[k]), k


@pytest.mark.parametrize("L", [1, 16, 100, 128, 200])
def test_equal_sequences(L):
    """[B, L, H] is the same as packed rows."""
    B, H = 5, 72
    s = make(B * L, H, B, torch.bfloat16, "sigmoid", L)
    cu = [L * i for i in range(B + 1)]
    want = run(s, cu, "sigmoid")
    t = {k: v.view(B, L, H) if k in ("gate", "value", "dy") else v for k, v in s.items()}
    got = run(t, cu, "sigmoid", packed=False)
    for k, v in want.items():
        assert torch.equal(v, got[k].reshape(v.shape)), k
    one = molt.gated_scan_fwd(s["gate"], s["value"])
    two = molt.gated_scan_fwd(s["gate"], s["value"], cu_seqlens=torch.tensor([0, B * L], dtype=torch.int32, device=dev()))
    assert torch.equal(one["y"], two["y"]) and one["final_state"].shape == (1, H)


def test_rows_outside_stay_as_they_were():
    T, H = 400, 64
    s = make(T, H, 2, torch.bfloat16, "sigmoid", 2)
    cu = torch.tensor([30, 130, 290], dtype=torch.int32, device=dev())
    out = torch.full((T, H), 9.0, dtype=torch.bfloat16, device=dev())
    s["gate"][:30] = s["value"][290:] = float("nan")     # nobody's
    got = molt.gated_scan_fwd(s["gate"], s["value"], cu_seqlens=cu, out=out, want_states=True)
    assert (out[:30] == 9).all() and (out[290:] == 9).all() and out[30:290].isfinite().all()
    assert got["final_state"].isfinite().all()
    g = molt.gated_scan_bwd(s["dy"], s["gate"], s["value"], got["states"], cu_seqlens=cu)
    for k in ("dgate", "dvalue"):
        assert (g[k][:30] == 0).all() and (g[k][290:] == 0).all() and g[k].isfinite().all()


@pytest.mark.parametrize("T", [60, 700])
def test_nothing_leaves_a_sequence(T):
    """Infinities, NaN and gates of plus and minus infinity in one sequence."""
    H = 66
    cu = [0, T // 3, T // 3, T // 2, T]
    s = make(T, H, 4, torch.float32, "sigmoid", T)
    want = run(s, cu, "sigmoid")
    bad = {k: v.clone() for k, v in s.items()}
    at = T // 3 + 2
    bad["value"][at, 0], bad["value"][at, 1], bad["dy"][at, 2] = INF, float("nan"), float("nan")
    bad["gate"][at, 3], bad["h0"][2, 4], bad["dfinal"][2, 5] = float("nan"), INF, float("nan")
    got = run(bad, cu, "sigmoid")
    for k in ("y", "dgate", "dvalue"):
        for a, b in ((0, T // 3), (T // 2, T)):
            assert torch.equal(got[k][a:b], want[k][a:b]), k
        assert not torch.equal(got[k][T // 3:T // 2], want[k][T // 3:T // 2])
    for k in ("final_state", "dinitial_state"):
        assert torch.equal(got[k][[0, 1, 3]], want[k][[0, 1, 3]]), k
    # a gate of +inf keeps the state, one of -inf replaces it
    s["gate"][:, 7], s["gate"][:, 8] = INF, -INF
    ref, out = reference(s, cu, "sigmoid"), run(s, cu, "sigmoid")
    for k in ("y", "dvalue"):
        check(out[k], ref[k], torch.float32, k)
    assert (out["dgate"][:, 7:9] == 0).all()


def test_log_gates_of_any_sign():
    """Growing channels, gates of 0 (a plain sum) and of minus infinity (nothing kept)."""
    T, H = 150, 64
    s = make(T, H, 1, torch.float32, "log", 3)
    s["gate"][:, 0], s["gate"][:, 1], s["gate"][:, 2], s["gate"][:, 3] = 0.02, 0.0, -INF, -1e-6
    s["gate"][:, 4], s["gate"][:, 5], s["gate"][:, 6] = 0.34999, -0.35001, -1e-30
    ref, out = reference(s, [0, T], "log"), run(s, [0, T], "log")
    fin = lambda r: (torch.nan_to_num(r[0]), torch.nan_to_num(r[1]))
    for k in ("y", "dvalue", "dgate"):
        check(out[k], fin(ref[k]), torch.float32, k)


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_channels_without_memory_beside_long_ones(dtype, kind):
    """Gates at which a is next to 0, in every other channel; their neighbours remember many rows.
    dgate in 16 bits: an a above 2^-7 may be off by 2^-24 twice over, 2^-16 of it."""
    T, H = 1000, 64
    s = make(T, H, 1, torch.float32, kind, 5)
    g = torch.Generator(device=dev()).manual_seed(6)
    s["gate"][:, ::2] = -3 - 30 * torch.rand(T, H // 2, device=dev(), generator=g)
    s["gate"][:, 1::2] = 9 + torch.rand(T, H // 2, device=dev(), generator=g) if kind == "sigmoid" else -1e-3
    for k in ("gate", "value", "dy"):
        s[k] = s[k].to(dtype)
    ref, out = reference(s, [0, T], kind), run(s, [0, T], kind)
    for k in ("y", "dvalue", "final_state", "dinitial_state"):
        check(out[k], ref[k], out[k].dtype, k)
    r, e = ref["dgate"]
    check(out["dgate"], (r, e + (r.abs() * 2.0 ** -16 if dtype != torch.float32 else 0)), dtype, "dgate")


@pytest.mark.parametrize("H,extra", [(64, 64), (65, 3), (128, 1), (320, 320)])
def test_strided_and_odd_rows(H, extra):
    """The halves of one projection, and rows that begin anywhere."""
    T = 200
    for dtype in DTYPES:
        s = make(T, H, 2, dtype, "sigmoid", H)
        cu = [0, 77, T]
        want = run(s, cu, "sigmoid")
        t = dict(s)
        for k in ("gate", "value", "dy"):
            wide = torch.full((T, H + extra + 1), 3.0, dtype=dtype, device=dev())
            wide[:, 1:H + 1] = s[k]
            t[k] = wide[:, 1:H + 1]
        got = run(t, cu, "sigmoid")
        for k, v in want.items():
            assert torch.equal(v, got[k]), (dtype, k)
    both = torch.cat([s["gate"], s["value"]], 1)
    got = molt.gated_scan_fwd(both[:, :H], both[:, H:], cu_seqlens=torch.tensor(cu, dtype=torch.int32, device=dev()))
    assert torch.equal(got["y"], molt.gated_scan_fwd(s["gate"], s["value"],
                                                     cu_seqlens=torch.tensor(cu, dtype=torch.int32, device=dev()))["y"])


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("B,H", [(1, 1), (3, 65), (64, 4096), (700, 320)])
def test_step(B, H, dtype, kind):
    """Steps, one after the other, are the rows of the scan."""
    n = 3
    s = make(n * B, H, B, dtype, kind, B)
    gate, value = s["gate"].view(B, n, H), s["value"].view(B, n, H)
    f, v = gate.double(), value.double()
    state = s["h0"].clone()
    for i in range(n):
        at = state.double()
        a = torch.sigmoid(f[:, i]) if kind == "sigmoid" else torch.exp(f[:, i])
        na = 1 - a
        ref = a * at + (na * v[:, i] if kind == "sigmoid" else v[:, i])
        e = TIMES * (E_NA * na * (at.abs() + v[:, i].abs()) + E_OP * (ref.abs() + at.abs() + v[:, i].abs()))
        out = molt.gated_scan_step(gate[:, i].contiguous(), value[:, i].contiguous(), state, kind=kind)
        check(out["state"], (ref, e), torch.float32, i)
        check(out["y"], (ref, e), dtype, i)
        strided = molt.gated_scan_step(gate[:, i], value[:, i], state.clone(), kind=kind)
        assert torch.equal(strided["y"], out["y"]) and torch.equal(strided["state"], out["state"])
        held = state.clone()
        inside = molt.gated_scan_step(gate[:, i], value[:, i], held, kind=kind, out_state=held)
        assert inside["state"] is held and torch.equal(held, out["state"])
        state = out["state"]
    whole = molt.gated_scan_fwd(gate, value, initial_state=s["h0"], kind=kind)
    ref = reference({**s, "dy": s["value"]}, [n * i for i in range(B + 1)], kind) if B * n < 300 else None
    if ref:
        check(whole["final_state"], ref["final_state"], torch.float32, "whole")


def test_gradients_against_differences():
    """Of the loss sum y dy + sum final dfinal in fp64, along directions."""
    T, H, cu = 90, 8, [0, 40, 41, 90]
    for kind in ("sigmoid", "log"):
        s = make(T, H, 3, torch.float32, kind, 7)
        out = run(s, cu, kind)
        gen = torch.Generator(device=dev()).manual_seed(1)

        def loss(m):
            a = torch.sigmoid(m["gate"]) if kind == "sigmoid" else torch.exp(m["gate"])
            b = (1 - a) * m["value"] if kind == "sigmoid" else m["value"]
            total = 0.0
            for n in range(3):
                h = m["h0"][n]
                for t in range(cu[n], cu[n + 1]):
                    h = a[t] * h + b[t]
                    total += float((h * m["dy"][t]).sum())
                total += float((h * m["dfinal"][n]).sum())
            return total

        d = {k: v.double() for k, v in s.items()}
        for name, grad in (("gate", "dgate"), ("value", "dvalue"), ("h0", "dinitial_state")):
            v = torch.randn(d[name].shape, device=dev(), generator=gen, dtype=torch.float64)
            eps = 1e-5
            diff = (loss({**d, name: d[name] + eps * v}) - loss({**d, name: d[name] - eps * v})) / (2 * eps)
            got = float((out[grad].double() * v).sum())
            # the difference's own error: eps^2 of third derivatives, and 1e-16 / eps of the loss
            assert abs(got - diff) <= 1e-4 * max(1.0, float(out[grad].norm())), (kind, name)


def test_no_rows():
    h0 = torch.randn(3, 64, device=dev())
    x = torch.empty(0, 64, dtype=torch.bfloat16, device=dev())
    cu = torch.zeros(4, dtype=torch.int32, device=dev())
    out = molt.gated_scan_fwd(x, x, initial_state=h0, cu_seqlens=cu, want_states=True)
    assert out["y"].shape == (0, 64) and torch.equal(out["final_state"], h0)
    g = molt.gated_scan_bwd(x, x, x, out["states"], initial_state=h0, cu_seqlens=cu, dfinal_state=2 * h0)
    assert torch.equal(g["dinitial_state"], 2 * h0)
    assert (molt.gated_scan_fwd(x, x, cu_seqlens=cu)["final_state"] == 0).all()
    e = molt.gated_scan_step(x, x, torch.empty(0, 64, device=dev()))
    assert e["y"].shape == (0, 64)


def test_bounds_that_descend_are_reported():
    """The kernels stay inside their tensors, the status word says so."""
    T, H = 300, 64
    s = make(T, H, 3, torch.bfloat16, "sigmoid", 1)
    assert molt.device_status() == 0
    for cu in ([0, 200, 100, 300], [0, 100, 200, 400], [-5, 100, 200, 300]):
        molt.gated_scan_fwd(s["gate"], s["value"], cu_seqlens=torch.tensor(cu, dtype=torch.int32, device=dev()))
        assert molt.device_status() == molt.DEV_FLAGS["unsorted_groups"]
    assert molt.device_status() == 0


@pytest.mark.parametrize("T", [5, 1000])
def test_in_a_captured_graph(T):
    H, B = 128, 3
    s = make(T, H, B, torch.bfloat16, "sigmoid", 1)
    cu = torch.tensor([0, 2, T // 2, T], dtype=torch.int32, device=dev())

    def calls():
        o = molt.gated_scan_fwd(s["gate"], s["value"], initial_state=s["h0"], cu_seqlens=cu, want_states=True)
        o.update(molt.gated_scan_bwd(s["dy"], s["gate"], s["value"], o["states"], initial_state=s["h0"], cu_seqlens=cu,
                                     dfinal_state=s["dfinal"]))
        o["step"] = molt.gated_scan_step(s["gate"][:B], s["value"][:B], o["final_state"])["y"]
        return o

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls()
    for seed, c in ((3, [0, 1, 1, T]), (4, [0, 0, T, T])):
        new = make(T, H, B, torch.bfloat16, "sigmoid", seed)
        for k in s:
            s[k].copy_(new[k])
        cu.copy_(torch.tensor(c, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        want = calls()
        for k, v in want.items():
            assert torch.equal(v, got[k]), k
