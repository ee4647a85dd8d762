"""Argument checks of the operators on the residual stream: every refusal happens on
the host, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300 import stream as S

FAKE = 0x1000   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


def desc(**kw):
    base = dict(T=4, H=64, x_stride=0, residual_stride=0, dy_stride=0, dtype=0, residual_dtype=0, param_dtype=2,
                gate_kind=0, res_scale=1.0, eps=1e-6, weight_offset=0.0)
    base.update(kw)
    return S.NormDesc(*[base[n] for n, _ in S.NormDesc._fields_])


def status(code):
    return molt.STATUS[code]


def norm_fwd(lib, d, x=FAKE, r=FAKE, w_post=None, gate=None, w_pre=FAKE, y=FAKE, r_out=FAKE):
    return status(lib.molt_residual_norm_fwd(ctypes.byref(d), x, r, w_post, gate, w_pre, y, r_out, None, None, None))


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), "MOLT_ERR_INVALID_ARG"), (dict(H=0), "MOLT_ERR_INVALID_ARG"),
    (dict(H=65537), "MOLT_ERR_UNSUPPORTED_SHAPE"), (dict(T=1 << 31), "MOLT_ERR_UNSUPPORTED_SHAPE"),
    (dict(dtype=3), "MOLT_ERR_INVALID_ARG"), (dict(residual_dtype=1), "MOLT_ERR_INVALID_ARG"),
    (dict(param_dtype=1), "MOLT_ERR_INVALID_ARG"), (dict(gate_kind=4), "MOLT_ERR_INVALID_ARG"),
    (dict(eps=-1.0), "MOLT_ERR_INVALID_ARG"), (dict(eps=float("nan")), "MOLT_ERR_INVALID_ARG"),
    (dict(res_scale=float("inf")), "MOLT_ERR_INVALID_ARG"), (dict(weight_offset=float("nan")), "MOLT_ERR_INVALID_ARG"),
    (dict(x_stride=63), "MOLT_ERR_INVALID_ARG"), (dict(residual_stride=-64), "MOLT_ERR_INVALID_ARG")])
def test_norm_refuses_descriptors(lib, kw, want):
    n0 = lib.molt_kernel_launches()
    assert norm_fwd(lib, desc(**kw)) == want
    assert lib.molt_residual_norm_bwd_workspace_bytes(ctypes.byref(desc(**kw))) == 0
    assert lib.molt_kernel_launches() == n0


def test_norm_refuses_missing_and_misaligned_pointers(lib):
    bad = "MOLT_ERR_INVALID_ARG"
    assert norm_fwd(lib, desc(), x=None) == bad
    assert norm_fwd(lib, desc(), y=None) == bad                     # w_pre without y
    assert norm_fwd(lib, desc(), w_pre=None, y=None, r_out=None) == bad
    assert norm_fwd(lib, desc(gate_kind=1)) == bad                  # gate missing
    assert norm_fwd(lib, desc(), x=FAKE + 1) == bad
    assert norm_fwd(lib, desc(residual_dtype=2), r=FAKE + 2) == bad
    assert status(lib.molt_residual_norm_fwd(None, *[FAKE] * 9, None)) == bad
    bwd = lambda d, **kw: status(lib.molt_residual_norm_bwd(ctypes.byref(d), *[kw.get(n, v) for n, v in (
        ("dy", FAKE), ("dr", FAKE), ("x", FAKE), ("r", FAKE), ("rstd_post", FAKE), ("rstd_pre", FAKE), ("w_post", FAKE),
        ("gate", None), ("w_pre", FAKE), ("dx", FAKE), ("dr_out", FAKE), ("dw_post", FAKE), ("dgate", None),
        ("dw_pre", FAKE))], 0, FAKE, 16, None))
    for kw in (dict(dy=None), dict(x=None), dict(r=None), dict(rstd_pre=None), dict(rstd_post=None), dict(dx=None),
               dict(dw_post=None), dict(dw_pre=None), dict(w_pre=None, dr=None), dict(dx=FAKE + 1),
               dict(rstd_pre=FAKE + 2)):
        assert bwd(desc(), **kw) == bad, kw
    assert bwd(desc(gate_kind=2), gate=FAKE) == bad                 # its gradient's buffer missing
    assert bwd(desc()) == "MOLT_ERR_WORKSPACE"


def test_embedding_refuses(lib):
    f = lambda E=FAKE, Et=0, tok=FAKE, T=4, H=8, V=9, scale=1.0, out=FAKE, ot=0: status(
        lib.molt_token_embedding(E, Et, tok, T, H, V, scale, out, ot, None))
    g = lambda d=FAKE, dt=0, tok=FAKE, T=4, H=8, V=9, scale=1.0, pad=-1, dE=FAKE, ot=0, acc=0: status(
        lib.molt_token_embedding_bwd(d, dt, tok, T, H, V, scale, pad, dE, ot, acc, FAKE, 16, None))
    bad, shape = "MOLT_ERR_INVALID_ARG", "MOLT_ERR_UNSUPPORTED_SHAPE"
    for kw in (dict(E=None), dict(tok=None), dict(out=None), dict(T=-1), dict(H=0), dict(V=0), dict(Et=3, ot=3),
               dict(ot=1), dict(Et=2, ot=0), dict(scale=float("nan")), dict(E=FAKE + 1), dict(out=FAKE + 2, ot=2),
               dict(tok=FAKE + 2)):
        assert f(**kw) == bad, kw
    assert f(T=1 << 31) == shape and f(V=1 << 31) == shape and f(H=65537) == shape
    for kw in (dict(d=None), dict(tok=None), dict(dE=None), dict(acc=1), dict(pad=9), dict(scale=float("inf")),
               dict(d=FAKE + 1), dict(ot=1), dict(T=-2)):
        assert g(**kw) == bad, kw
    assert f(T=0) == "MOLT_OK"
    assert lib.molt_token_embedding_bwd_workspace_bytes(10, 0, 5) == 0


def test_workspaces_never_shrink_as_tokens_grow(lib):
    Ts = sorted({max(0, 1024 * k + d) for k in (*range(0, 70), *range(70, 400, 13)) for d in (-1, 0, 1, 8)})
    for H in (1, 64, 320, 5120):
        last = 0
        for T in Ts:
            n = lib.molt_token_embedding_bwd_workspace_bytes(T, H, 32000)
            assert n >= last
            last = n
        sizes = [lib.molt_residual_norm_bwd_workspace_bytes(ctypes.byref(desc(T=T, H=H))) for T in Ts]
        assert sizes == sorted(sizes)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="CUDA"):
        molt.residual_norm_fwd(x, w_pre=torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="gate"):
        molt.residual_norm_fwd(x, gate=torch.ones(5), w_pre=torch.ones(64))
    with pytest.raises(ValueError, match="shape"):
        molt.residual_norm_fwd(x, residual=torch.zeros(4, 32, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="w_pre"):
        molt.residual_norm_fwd(x, w_pre=torch.ones(65))
    with pytest.raises(TypeError, match="one type"):
        molt.residual_norm_fwd(x, w_post=torch.ones(64), w_pre=torch.ones(64, dtype=torch.bfloat16))
    with pytest.raises(TypeError, match="w_pre"):
        molt.residual_norm_fwd(x, w_pre=torch.ones(64, dtype=torch.float16))
    with pytest.raises(TypeError, match="CUDA"):
        molt.token_embedding(torch.zeros(9, 8), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError, match="CUDA"):
        molt.token_embedding_bwd(torch.zeros(3, 8), torch.zeros(3, dtype=torch.int32), 9, workspace=torch.empty(1))
    with pytest.raises(ValueError, match="tokens"):
        molt.token_embedding_bwd(torch.zeros(3, 8), torch.zeros(4, dtype=torch.int32), 9)
    with pytest.raises(TypeError, match="float16 or float32"):
        S._dtype_code(torch.float64, "x")
