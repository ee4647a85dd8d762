"""Cross entropy over the LM head against the formulas in fp64.

Tolerances, before any run, are those of the LM head's other calls (tests/parity.py):
logp and lse within 2e-3, the loss within 1e-3 of max(its size, sum w / D), gradients
within 2e-2 of the largest entry with a cosine of at least 0.9999 (products of a
gradient rounded to bf16, 2^-8, with bf16 operands; a bf16 dW rounds once more)."""
import numpy as np
import pytest
import torch

import paper_2607_21653_gb300 as molt
from parity import LOGP_ATOL, LOSS_RTOL, assert_grad_close, dev

pytestmark = pytest.mark.gpu
IGN = -100


def make(T, H, V, masked=0.0, seed=0, known=True):
    g = torch.Generator().manual_seed(seed + T + 3 * H + 7 * V)
    W = (torch.randn(V, H, generator=g) * 0.02).to(torch.bfloat16)
    x = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    h = torch.randn(T, H, generator=g)
    if known:   # half of the targets are predicted
        h = h + (torch.rand(T, generator=g) < 0.5).float()[:, None] * W[x.long()].float() * (6.0 / (H * 4e-4))
    x[torch.rand(T, generator=g) < masked] = IGN
    w = 0.25 + torch.rand(T, generator=g)
    return h.to(torch.bfloat16).to(dev()), W.to(dev()), x.to(dev()), w.to(dev())


def reference(h, W, x, w=None, e=0.0, c=0.0, denom=0.0, ignore=IGN):
    T, V = h.shape[0], W.shape[0]
    h, W = h.double(), W.double()
    x = x.long()   # an int32 compare would wrap a large ignore_index
    act = x != ignore
    ok = act & (x >= 0) & (x < V)
    xi = torch.where(ok, x, torch.zeros_like(x))
    z = h @ W.t()
    lse = torch.logsumexp(z, 1)
    zx = z.gather(1, xi[:, None])[:, 0]
    l = lse - (1 - e) * zx - e * z.mean(1) + c * lse * lse
    D = denom if denom > 0 else float(act.sum())
    wt = ok.double() * (1.0 if w is None else w.double())
    coef = wt / D if D > 0 else torch.zeros_like(wt)
    g = torch.softmax(z, 1) * (1 + 2 * c * lse)[:, None] - e / V
    g.scatter_add_(1, xi[:, None], torch.full((T, 1), -(1 - e), dtype=torch.float64, device=h.device))
    g = g * coef[:, None]
    return {"loss": (coef * l).sum(), "size": max(float((coef * l.abs()).sum()), float(coef.sum())), "logp": torch.where(ok, zx - lse, 0.0 * lse),
            "lse": torch.where(act, lse, 0.0 * lse), "dhidden": g @ W, "dW": g.t() @ h, "act": act, "nll": ((lse - zx) * ok).sum(),
            "lse2": (lse * lse * ok).sum(), "D": D}


def check(out, ref, grad=True):
    assert (out["logp"].double() - ref["logp"]).abs().max() <= LOGP_ATOL
    assert (out["lse"].double() - ref["lse"]).abs().max() <= LOGP_ATOL
    assert (out["logp"][~ref["act"]] == 0).all() and (out["lse"][~ref["act"]] == 0).all()
    assert abs(float(out["loss"]) - float(ref["loss"])) <= LOSS_RTOL * ref["size"]
    st = molt.cross_entropy_stats(out["stats"])
    assert st["n_active"] == int(ref["act"].sum()) and st["denom"] == ref["D"]
    assert abs(st["loss"] - float(out["loss"])) <= 1e-6 * abs(st["loss"])
    assert abs(st["sum_nll"] - float(ref["nll"])) <= LOGP_ATOL * max(1, st["n_active"])
    assert abs(st["sum_lse_sq"] - float(ref["lse2"])) <= 2 * LOGP_ATOL * max(1.0, float(ref["lse2"]))
    if not grad:
        return
    assert (out["dhidden"][~ref["act"]] == 0).all()
    for k in ("dhidden", "dW"):
        assert_grad_close(out[k].double().cpu().numpy(), ref[k].cpu().numpy(), k)


SHAPES = [(1, 64, 2), (1, 256, 5000), (3, 64, 257), (100, 128, 1000), (129, 192, 255), (256, 256, 256), (257, 320, 4097),
          (700, 512, 3000), (1031, 896, 5003), (2100, 256, 2600), (4500, 320, 700), (600, 2048, 9000), (300, 1088, 12000)]


@pytest.mark.parametrize("dW_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,V", SHAPES)
def test_plain(T, H, V, dW_dtype):
    h, W, x, _ = make(T, H, V, 0.2 if T > 3 else 0.0)
    out = molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=dW_dtype)
    assert out["dW"].dtype == dW_dtype
    check(out, reference(h, W, x))
    only = molt.cross_entropy_fwd(h, W, x)
    for k in ("loss", "logp", "lse", "stats"):
        assert torch.equal(only[k], out[k]), k
    assert molt.device_status() == 0


@pytest.mark.parametrize("T,H,V", [(1, 64, 2), (100, 128, 1000), (257, 320, 4097), (1031, 896, 5003), (4500, 256, 3000)])
@pytest.mark.parametrize("e,c,weighted,denom", [(0.1, 0.0, False, 0.0), (0.0, 1e-2, False, 0.0), (0.2, 1e-3, True, 0.0),
                                               (0.0, 0.0, True, 777.0), (1.0, 0.0, False, 0.0)])
def test_terms(T, H, V, e, c, weighted, denom):
    h, W, x, w = make(T, H, V, 0.3 if T > 3 else 0.0, seed=1)
    w = w if weighted else None
    if w is not None and T > 3:
        w[::5] = 0.0
    kw = dict(token_weight=w, label_smoothing=e, z_loss=c, denom=denom)
    ref = reference(h, W, x, w, float(np.float32(e)), float(np.float32(c)), denom)
    check(molt.cross_entropy_fwd(h, W, x, **kw), ref, grad=False)
    check(molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=torch.bfloat16, **kw), ref)
    assert molt.device_status() == 0


@pytest.mark.parametrize("T,H,V,masked", [(4500, 1024, 3001, 0.0), (9000, 1088, 2000, 0.15), (8700, 1024, 1500, 0.0),
                                          (4500, 960, 1501, 0.0), (4500, 1152, 700, 0.5)])
def test_rounded_weight_gradient(T, H, V, masked):
    """bf16 dW of as many tokens as one chunk takes, of more and of fewer."""
    h, W, x, _ = make(T, H, V, masked, seed=9)
    out = molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=torch.bfloat16, label_smoothing=0.05)
    check(out, reference(h, W, x, e=float(np.float32(0.05))))
    assert molt.device_status() == 0


@pytest.mark.parametrize("spread", [1.0, 40.0, 2000.0])
@pytest.mark.parametrize("H", [576, 640])
def test_logits_far_apart(H, spread):
    """Rows whose logits lie up to `spread` apart, at widths whose logits are formed again
    and kept.  The products' fp32 sums of H terms of up to z / 4 are good to 1e-5 z at the
    most, so logp is held to that where it is more than LOGP_ATOL."""
    T, V = 300, 1300
    h, W, x, _ = make(T, H, V, 0.1, seed=11, known=False)
    h = (h.float() * (torch.rand(T, 1, device=h.device, generator=torch.Generator(device=h.device).manual_seed(1)) * spread)).to(torch.bfloat16)
    out, ref = molt.cross_entropy_fwd_bwd(h, W, x), reference(h, W, x)
    size = float((h.double() @ W.double().t()).abs().max())
    assert (out["logp"].double() - ref["logp"]).abs().max() <= max(LOGP_ATOL, 1e-5 * size)
    assert abs(float(out["loss"]) - float(ref["loss"])) <= LOSS_RTOL * ref["size"]
    for k in ("dhidden", "dW"):
        assert_grad_close(out[k].double().cpu().numpy(), ref[k].cpu().numpy(), k)


def test_a_column_of_minus_infinity():
    """A column whose logit is -inf in every row: no part of the others' sums; a row that has
    it as its target has logp -inf and makes the loss +inf."""
    h, W, x, _ = make(300, 128, 700, seed=14, known=False)
    h[:, 5] = h[:, 5].abs() + 0.1
    W[7, 5] = float("-inf")
    x[x == 7] = 8
    keep = torch.arange(700, device=h.device) != 7
    xr = torch.where(x > 7, x - 1, x)
    for targets, bad in ((x, False), (torch.where(torch.arange(300, device=h.device) == 17, 7, x).to(torch.int32), True)):
        out = molt.cross_entropy_fwd(h, W, targets)
        ref = reference(h, W[keep], xr)
        rows = torch.arange(300, device=h.device) != 17
        assert (out["logp"].double() - ref["logp"])[rows].abs().max() <= LOGP_ATOL
        assert (out["lse"].double() - ref["lse"]).abs().max() <= LOGP_ATOL
        if bad:
            assert out["logp"][17] == float("-inf") and out["loss"][0] == float("inf")
        else:
            assert abs(float(out["loss"]) - float(ref["loss"])) <= LOSS_RTOL * ref["size"]


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_kept_logits_show_a_bad_row(value):
    """As without keeping: the row's dhidden and dW are NaN, the other rows' dhidden is not."""
    h, W, x, _ = make(300, 640, 700, seed=12)
    h[17, 3] = value
    out = molt.cross_entropy_fwd_bwd(h, W, x)
    assert torch.isnan(out["dhidden"][17]).all() and torch.isnan(out["dW"]).all() and torch.isnan(out["loss"]).all()
    rest = torch.arange(300, device=h.device) != 17
    good = molt.cross_entropy_fwd_bwd(h[rest], W, x[rest], denom=300.0)
    # an upper tile's K blocks may hold the bad row's zeros only: rows are independent
    assert torch.isfinite(out["dhidden"][rest]).all()
    assert (out["dhidden"][rest].float() - good["dhidden"].float()).abs().max() <= 2e-2 * good["dhidden"].float().abs().max()


def test_more_logits_than_are_kept():
    """The last token tiles' logits are formed again; against two calls of half the rows,
    which keep all of theirs (each side is good to 2e-2, so they agree to 4e-2)."""
    T, H, V = 8300, 640, 262149
    h, W, x, _ = make(T, H, V, seed=13)
    out = molt.cross_entropy_fwd_bwd(h, W, x, denom=float(T))
    dW = None
    for rows in (slice(0, 4150), slice(4150, T)):
        part = molt.cross_entropy_fwd_bwd(h[rows], W, x[rows], denom=float(T), dW=dW, accumulate_dW=dW is not None)
        dW = part["dW"]
        assert (out["logp"][rows] - part["logp"]).abs().max() <= 2 * LOGP_ATOL
        far = (out["dhidden"][rows].float() - part["dhidden"].float()).abs().max()
        assert far <= 4e-2 * part["dhidden"].float().abs().max()
    assert (out["dW"] - dW).abs().max() <= 4e-2 * dW.abs().max()
    assert molt.device_status() == 0


def test_one_column_has_no_loss():
    h, W, x, _ = make(10, 64, 1, known=False)
    out = molt.cross_entropy_fwd_bwd(h, W, x)
    # p - 1 is the rounding of e^(z - lse) alone
    assert out["loss"].abs() <= 1e-5 and out["dW"].abs().max() <= 1e-4 and out["dhidden"].abs().max() <= 1e-4


def test_every_target_ignored():
    h, W, x, _ = make(300, 256, 900)
    x.fill_(IGN)
    base = torch.ones(900, 256, device=dev())
    out = molt.cross_entropy_fwd_bwd(h, W, x, dW=base, accumulate_dW=True)
    assert molt.device_status() == molt.DEV_FLAGS["zero_denom"]
    assert float(out["loss"]) == 0 and (out["dhidden"] == 0).all() and (base == 1).all() and (out["lse"] == 0).all()
    for dt in (torch.float32, torch.bfloat16):
        out = molt.cross_entropy_fwd_bwd(h, W, x, denom=5.0, dW_dtype=dt, dW=torch.full((900, 256), 3.0, dtype=dt, device=dev()))
        assert (out["dW"] == 0).all() and molt.device_status() == 0
    assert molt.cross_entropy_stats(molt.cross_entropy_fwd(h, W, x, denom=5.0)["stats"])["n_active"] == 0


def test_no_tokens():
    h, W, x, _ = make(4, 64, 30)
    out = molt.cross_entropy_fwd_bwd(h[:0], W, x[:0], dW_dtype=torch.bfloat16)
    assert float(out["loss"]) == 0 and (out["dW"] == 0).all() and out["dhidden"].shape == (0, 64)


def test_targets_out_of_range():
    """They count in the denominator and have no loss and no gradient."""
    h, W, x, _ = make(200, 128, 500, 0.1)
    x[3], x[100], x[199] = -1, 500, 2**31 - 1
    for e in (0.0, 0.1):
        out = molt.cross_entropy_fwd_bwd(h, W, x, label_smoothing=e)
        assert molt.device_status() == molt.DEV_FLAGS["token_range"]
        check(out, reference(h, W, x, e=float(np.float32(e))))
        assert (out["dhidden"][[3, 100, 199]] == 0).all()


@pytest.mark.parametrize("ignore", [0, 7, -1, 2**40])
def test_ignore_index(ignore):
    h, W, x, _ = make(400, 192, 20, seed=2)
    if ignore == -1:
        x[50:90] = -1
    check(molt.cross_entropy_fwd_bwd(h, W, x, ignore_index=ignore), reference(h, W, x, ignore=ignore))
    assert molt.device_status() == 0


def test_first_and_last_rows_ignored():
    """Packed rows in the middle of whole tiles of ignored ones."""
    h, W, x, _ = make(3000, 256, 1500, seed=3)
    x[:1111] = IGN
    x[2500:] = IGN
    check(molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=torch.bfloat16), reference(h, W, x))


def test_microbatches_add_up():
    h, W, x, _ = make(1500, 256, 2000, 0.2, seed=4)
    ref = reference(h, W, x)
    dW = torch.empty(2000, 256, device=dev())
    loss, dh = 0.0, []
    for i, (a, b) in enumerate([(0, 700), (700, 701), (701, 1500)]):
        out = molt.cross_entropy_fwd_bwd(h[a:b], W, x[a:b].contiguous(), denom=ref["D"], dW=dW, accumulate_dW=i > 0)
        loss += float(out["loss"])
        dh.append(out["dhidden"])
    assert abs(loss - float(ref["loss"])) <= LOSS_RTOL * ref["size"]
    assert_grad_close(torch.cat(dh).double().cpu().numpy(), ref["dhidden"].cpu().numpy(), "dhidden")
    assert_grad_close(dW.double().cpu().numpy(), ref["dW"].cpu().numpy(), "dW")


def test_same_gradient_as_the_policy_loss():
    """With behaviour = current log-probs and advantages of 1 the clipped surrogate's
    gradient is the cross entropy's: ratio 1 (to the rounding of expf(0)), unclipped."""
    h, W, x, _ = make(900, 512, 3000, seed=5)
    ce = molt.cross_entropy_fwd_bwd(h, W, x)
    pl = molt.policy_loss_fwd_bwd(h, W, x, ce["logp"], torch.ones(900, device=dev()))
    assert (ce["logp"] - pl["logp"]).abs().max() <= LOGP_ATOL
    assert_grad_close(ce["dW"].cpu().numpy(), pl["dW"].cpu().numpy(), "dW")
    assert_grad_close(ce["dhidden"].float().cpu().numpy(), pl["dhidden"].float().cpu().numpy(), "dhidden")


@pytest.mark.parametrize("e,c", [(0.0, 0.0), (0.1, 1e-2)])
def test_gradient_by_differences(e, c):
    """The loss along a step in the hidden states and one in W, against the gradients.  The
    gradients are good to 2e-2 (above) of |gradient| |step|; the loss is fp64 sums of rows
    good to a few 1e-6, on differences of 1e-2; the central difference's own error is of
    third order: 3e-2 of |gradient| |step| covers them."""
    T, H, V = 96, 128, 400
    h, W, x, _ = make(T, H, V, 0.2, seed=6)
    kw = dict(label_smoothing=e, z_loss=c)
    out = molt.cross_entropy_fwd_bwd(h, W, x, **kw)
    loss = lambda h, W: molt.cross_entropy_stats(molt.cross_entropy_fwd(h, W, x, **kw)["stats"])["loss"]
    g = torch.Generator(device=dev()).manual_seed(1)
    for name, grad in (("h", out["dhidden"]), ("W", out["dW"])):
        base = h if name == "h" else W
        # along the gradient, so that the difference is not lost in rounding
        step = grad.float() / grad.float().norm() * (2.0 if name == "h" else 0.3)
        step = step + 0.2 * step.norm() / base.numel()**0.5 * torch.randn(step.shape, device=dev(), generator=g)
        plus, minus = (base.float() + step).to(torch.bfloat16), (base.float() - step).to(torch.bfloat16)
        real = (plus.double() - minus.double())
        got = loss(plus, W) - loss(minus, W) if name == "h" else loss(h, plus) - loss(h, minus)
        want = float((grad.double() * real).sum())
        assert abs(got - want) <= 3e-2 * float(grad.double().norm() * real.norm()), (name, got, want)


def test_reproducible_outputs_of_the_forward():
    h, W, x, w = make(3000, 320, 5000, 0.3, seed=7)
    a, b = (molt.cross_entropy_fwd(h, W, x, token_weight=w, label_smoothing=0.1, z_loss=1e-4) for _ in range(2))
    for k in ("loss", "stats"):
        assert torch.equal(a[k], b[k]), k


def test_non_finite_hidden_shows_in_its_row():
    h, W, x, _ = make(300, 128, 700, seed=8)
    ok = molt.cross_entropy_fwd(h, W, x)
    h[17, 3] = float("nan")
    out = molt.cross_entropy_fwd(h, W, x)
    assert torch.isnan(out["logp"][17]) and torch.isnan(out["loss"]).all()
    rest = [t for t in range(300) if t != 17]
    assert torch.equal(out["logp"][rest], ok["logp"][rest])


def test_other_stream_workspace_and_poison():
    h, W, x, _ = make(700, 320, 3000, 0.2, seed=9)
    ref = reference(h, W, x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=torch.bfloat16)
    torch.cuda.current_stream().wait_stream(s)
    check(out, ref)
    L = molt.load()
    n = L.molt_cross_entropy_workspace_bytes(700, 320, 3000, 1, 0)
    check(molt.cross_entropy_fwd_bwd(h, W, x, dW_dtype=torch.bfloat16,
                                     workspace=torch.full((n,), 255, dtype=torch.uint8, device=dev())), ref)
    with pytest.raises(molt.MoltError) as err:
        molt.cross_entropy_fwd_bwd(h, W, x, workspace=torch.empty(4096, dtype=torch.uint8, device=dev()))
    assert err.value.status == 9


def test_in_a_captured_graph():
    h, W, x, _ = make(500, 256, 2000, 0.2, seed=10)
    ref = reference(h, W, x)
    ws = torch.empty(molt.load().molt_cross_entropy_workspace_bytes(500, 256, 2000, 1, 2), dtype=torch.uint8, device=dev())
    molt.cross_entropy_fwd_bwd(h, W, x, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = molt.cross_entropy_fwd_bwd(h, W, x, workspace=ws)
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    check(out, ref)
