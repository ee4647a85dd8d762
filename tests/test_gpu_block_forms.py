"""Forms of the operators inside a block that the other files leave out: gelu with kept products and relu with formed
ones, equal sequences in every type, and products of tokens and channels past 2^31 elements.  Tolerances are those of
test_gpu_gated_ffn.py, element by element; the weights' gradients of the long call against two halves of it: what is
summed is rounded alike but where a product's K is cut in another way, and a rounding more, 2^-8 of the norm."""
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import dev
from test_gpu_gated_ffn import BF, F32, HF, U, bwd_reference, check, fwd_reference, inputs, rounded
from test_gpu_gated_scan import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("act,kept", [("gelu", True), ("relu", False)])
@pytest.mark.parametrize("T,H,F", [(1, 64, 64), (9, 512, 1000), (33, 1024, 264), (257, 328, 264), (1031, 896, 2392)])
def test_gradients(T, H, F, act, kept, dtype):
    s = inputs(T, H, F, dtype, T + F)
    w = (s["x"], s["w_gate"], s["w_up"], s["w_down"])
    k = molt.gated_ffn_fwd(*w, activation=act, keep=True) if kept else {"gate": None, "up": None}
    out = molt.gated_ffn_bwd(s["dy"], *w, gate=k["gate"], up=k["up"], activation=act, dw_dtype=F32)
    for name, (r, e) in bwd_reference(s, act, dtype, k["gate"], k["up"]).items():
        if name == "dx":
            check(out[name], r, rounded(r, e, dtype), dtype, name)
        else:
            check(out[name], r, e + 2.0**-24 * r.abs(), F32, name)


@pytest.mark.parametrize("kind", ["sigmoid", "log"])
@pytest.mark.parametrize("dtype", [HF, F32])
@pytest.mark.parametrize("L,H", [(1, 72), (17, 65), (128, 72), (200, 64)])
def test_equal_sequences(L, H, dtype, kind):
    B = 5
    s = make(B * L, H, B, dtype, kind, L)
    want = run(s, [L * i for i in range(B + 1)], kind)
    t = {k: v.view(B, L, H) if k in ("gate", "value", "dy") else v for k, v in s.items()}
    got = run(t, [L * i for i in range(B + 1)], kind, packed=False)
    for k, v in want.items():
        assert torch.equal(v, got[k].reshape(v.shape)), k


@pytest.mark.parametrize("kept", [True, False])
def test_more_elements_than_31_bits_count(kept):
    T, H, F = 262184, 64, 8200
    at = (1 << 31) // F
    assert T * F > 1 << 31 and at + 40 < T - 48
    s = inputs(T, H, F, BF, 1)
    w = (s["w_gate"], s["w_up"], s["w_down"])
    k = molt.gated_ffn_fwd(s["x"], *w, keep=True) if kept else {"gate": None, "up": None}
    out = molt.gated_ffn_bwd(s["dy"], s["x"], *w, gate=k["gate"], up=k["up"])
    for rows in (slice(0, 48), slice(at - 40, at + 40), slice(T - 48, T)):
        part = {**s, "x": s["x"][rows], "dy": s["dy"][rows]}
        if kept:
            for name, (r, b) in fwd_reference(part, "silu", BF).items():
                check(k[name][rows], r, b, BF, name)
        r, e = bwd_reference(part, "silu", BF, k["gate"][rows] if kept else None, k["up"][rows] if kept else None)["dx"]
        check(out["dx"][rows], r, rounded(r, e, BF), BF, "dx")
    total = None
    for rows in (slice(0, T // 2), slice(T // 2, T)):
        more = (k["gate"][rows], k["up"][rows]) if kept else (None, None)
        half = molt.gated_ffn_bwd(s["dy"][rows], s["x"][rows], *w, *more)
        total = half if total is None else {n: t + half[n] for n, t in total.items() if n != "dx"}
    for name, t in total.items():
        assert float((out[name] - t).norm()) <= U[BF] * float(t.norm()), name
    assert molt.device_status() == 0
