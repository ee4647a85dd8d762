"""Argument checks of the cross entropy: every refusal happens on the host."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300.cross_entropy import CrossEntropyOptions

FAKE = 0x1000   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


def call(lib, opts=None, **kw):
    a = dict(h=FAKE, W=FAKE, x=FAKE, w=None, T=16, H=64, V=32, denom=0.0, loss=FAKE, dh=FAKE, dW=FAKE, dt=2, acc=0, ws=FAKE,
             n=16)
    a.update(kw)
    o = None if opts is None else ctypes.byref(CrossEntropyOptions(*opts))
    st = lib.molt_cross_entropy_fwd_bwd(a["h"], a["W"], a["x"], a["w"], a["T"], a["H"], a["V"], a["denom"], o, a["loss"],
                                        a["dh"], a["dW"], a["dt"], a["acc"], None, None, None, a["ws"], a["n"], None)
    return molt.STATUS[st]


@pytest.mark.parametrize("kw", [dict(h=None), dict(W=None), dict(x=None), dict(loss=None), dict(dh=None), dict(dW=None),
                                dict(h=FAKE + 2), dict(W=FAKE + 8), dict(dh=FAKE + 2), dict(dW=FAKE + 4), dict(T=-1),
                                dict(V=0), dict(denom=float("nan")), dict(dt=1), dict(dt=3), dict(dt=0, acc=1),
                                dict(opts=(-100, -0.1, 0.0)), dict(opts=(-100, 1.1, 0.0)), dict(opts=(-100, 0.0, -1.0)),
                                dict(opts=(-100, float("nan"), 0.0)), dict(opts=(-100, 0.0, float("inf")))])
def test_refuses(lib, kw):
    n0 = lib.molt_kernel_launches()
    assert call(lib, **kw) == "MOLT_ERR_INVALID_ARG"
    assert lib.molt_kernel_launches() == n0


def test_refuses_shapes(lib):
    assert call(lib, H=100) == "MOLT_ERR_UNSUPPORTED_SHAPE"
    assert call(lib, T=1 << 31) == "MOLT_ERR_UNSUPPORTED_SHAPE"
    assert lib.molt_cross_entropy_workspace_bytes(16, 100, 32, 1, 2) == 0
    fwd = lib.molt_cross_entropy_fwd_bwd
    assert fwd is not None
    st = lib.molt_cross_entropy_fwd(FAKE, FAKE, None, None, 16, 64, 32, 0.0, None, FAKE, None, None, None, FAKE, 16, None)
    assert molt.STATUS[st] == "MOLT_ERR_INVALID_ARG"


@pytest.mark.parametrize("H", [64, 256, 320, 1024, 4096])
def test_workspace_never_shrinks_as_tokens_grow(lib, H):
    Ts = sorted({max(0, 128 * k + d) for k in (*range(0, 64), *range(64, 600, 7)) for d in (-1, 0, 1)})
    for V in (1, 4096, 5000, 32000, 151936):
        for back, dt in ((0, 2), (1, 2), (1, 0)):
            sizes = [lib.molt_cross_entropy_workspace_bytes(T, H, V, back, dt) for T in Ts]
            assert sizes == sorted(sizes) and sizes[-1] > 0


@pytest.mark.parametrize("V", [1, 151936, (1 << 31) - 300])
def test_workspace_of_the_largest_calls(lib, V):
    """Sizes whose products pass 64 bits where they are not held back."""
    Ts = [1 << k for k in range(20, 31)] + [(1 << 31) - 1000]
    sizes = [lib.molt_cross_entropy_workspace_bytes(T, 1024, V, 1, 2) for T in Ts]
    assert sizes == sorted(sizes)
    assert all(T * 1024 * 2 < n < 1 << 62 for T, n in zip(Ts, sizes))


def test_binding_refuses():
    h, W, x = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(9, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="weight"):
        molt.cross_entropy_fwd(h, W[:, :32], x)
    with pytest.raises(ValueError, match="targets"):
        molt.cross_entropy_fwd(h, W, x[:3])
    with pytest.raises(ValueError, match="token_weight"):
        molt.cross_entropy_fwd(h, W, x, token_weight=torch.ones(5))
    with pytest.raises(ValueError, match="dW"):
        molt.cross_entropy_fwd_bwd(h, W, x, dW=torch.zeros(8, 64))
    with pytest.raises(TypeError, match="CUDA"):
        molt.cross_entropy_fwd(h, W, x, workspace=torch.empty(1))
