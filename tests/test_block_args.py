"""Argument checks of the operators inside a block: every refusal happens on the host, before
anything is launched."""
import ctypes

import pytest
import torch

import paper_2607_21653_gb300 as molt
from paper_2607_21653_gb300 import blocks as B

FAKE = 1 << 20   # never dereferenced: every call below fails validation first
BAD, SHAPE = "MOLT_ERR_INVALID_ARG", "MOLT_ERR_UNSUPPORTED_SHAPE"


@pytest.fixture(scope="module")
def lib():
    molt.build()
    return molt.load()


def make(cls, base, kw):
    v = {**base, **kw}
    return cls(*[v[n] for n, _ in cls._fields_])


def ffn(**kw):
    return make(B.FfnDesc, dict(T=4, H=64, F=128, x_stride=0, w_gate_stride=0, w_up_stride=0, w_down_stride=0, dy_stride=0,
                                dtype=0, activation=0), kw)


def scan(**kw):
    return make(B.ScanDesc, dict(T=4, H=64, B=2, gate_stride=0, value_stride=0, dy_stride=0, dtype=0, form=0,
                                 fill_outside=0), kw)


def drop(**kw):
    return make(B.DropoutDesc, dict(T=4, H=64, x_stride=0, residual_stride=0, first_row=0, seed=1, offset=0, p=0.1,
                                    res_scale=1.0, dtype=0, out_dtype=0), kw)


def status(code):
    return molt.STATUS[code]


def ffn_fwd(lib, d, **kw):
    names = ("x", "w_gate", "w_up", "w_down", "y", "gate_out", "up_out", "ws")
    ptr = {**{n: FAKE * (i + 1) for i, n in enumerate(names)}, "gate_out": None, "up_out": None, **kw}
    return status(lib.molt_gated_ffn_fwd(ctypes.byref(d), *[ptr[n] for n in names], 16, None))


def ffn_bwd(lib, d, dw_dtype=2, accumulate=0, **kw):
    names = ("dy", "x", "w_gate", "w_up", "w_down", "gate", "up", "dx", "dw_gate", "dw_up", "dw_down")
    ptr = {**{n: FAKE * (i + 1) for i, n in enumerate(names)}, **kw}
    return status(lib.molt_gated_ffn_bwd(ctypes.byref(d), *[ptr[n] for n in names], dw_dtype, accumulate, FAKE, 16, None))


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), BAD), (dict(H=0), BAD), (dict(F=0), BAD), (dict(dtype=2), BAD), (dict(dtype=-1), BAD),
    (dict(activation=3), BAD), (dict(activation=-1), BAD), (dict(H=60), SHAPE), (dict(F=100), SHAPE),
    (dict(H=(1 << 17) + 8), SHAPE), (dict(F=(1 << 17) + 8), SHAPE), (dict(T=(1 << 24) + 1), SHAPE),
    (dict(x_stride=56), BAD), (dict(w_gate_stride=-64), BAD), (dict(w_down_stride=64), BAD), (dict(w_up_stride=68), SHAPE),
    (dict(dy_stride=1 << 32), SHAPE)])
def test_ffn_refuses_descriptors(lib, kw, want):
    n0 = lib.molt_kernel_launches()
    assert ffn_fwd(lib, ffn(**kw)) == want
    assert ffn_bwd(lib, ffn(**kw)) == want
    d = ffn(**kw)
    assert lib.molt_gated_ffn_fwd_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.molt_gated_ffn_bwd_workspace_bytes(ctypes.byref(d), 1) == 0
    assert lib.molt_kernel_launches() == n0


def test_ffn_refuses_pointers(lib):
    for n in ("x", "w_gate", "w_up", "w_down", "y"):
        assert ffn_fwd(lib, ffn(), **{n: None}) == BAD, n
        assert ffn_fwd(lib, ffn(), **{n: FAKE + 8}) == BAD, n
    assert ffn_fwd(lib, ffn(), gate_out=FAKE) == BAD                     # up_out missing
    assert ffn_fwd(lib, ffn(), gate_out=FAKE, up_out=FAKE + 2) == BAD
    assert ffn_fwd(lib, ffn()) == "MOLT_ERR_WORKSPACE"
    assert ffn_fwd(lib, ffn(T=0), x=None, y=None) == "MOLT_OK"
    for n in ("dy", "x", "w_gate", "w_up", "w_down", "dx", "dw_gate", "dw_up", "dw_down", "gate", "up"):
        assert ffn_bwd(lib, ffn(), **{n: None}) == BAD, n
        assert ffn_bwd(lib, ffn(), **{n: FAKE + 4}) == BAD, n
    assert ffn_bwd(lib, ffn(), dw_dtype=1) == BAD
    assert ffn_bwd(lib, ffn(), dw_dtype=0, accumulate=1) == BAD
    assert ffn_bwd(lib, ffn()) == "MOLT_ERR_WORKSPACE"
    assert status(lib.molt_gated_ffn_fwd(None, *[FAKE] * 8, 16, None)) == BAD


def test_ffn_workspaces_never_shrink_as_tokens_grow(lib):
    """A buffer for the largest batch serves every smaller one."""
    Ts = sorted({max(0, 64 * k + d) for k in (*range(0, 40), *range(40, 400, 11)) for d in (-1, 0, 1, 8)})
    for H, F in ((64, 64), (896, 2392), (4096, 10944), (5120, 256)):
        for q in (lambda d: lib.molt_gated_ffn_fwd_workspace_bytes(d), lambda d: lib.molt_gated_ffn_bwd_workspace_bytes(d, 0),
                  lambda d: lib.molt_gated_ffn_bwd_workspace_bytes(d, 1)):
            sizes = [q(ctypes.byref(ffn(T=T, H=H, F=F))) for T in Ts]
            assert sizes == sorted(sizes) and sizes[0] > 0


def scan_fwd(lib, d, **kw):
    names = ("gate", "value", "h0", "cu", "y", "final", "states")
    ptr = {**{n: FAKE * (i + 1) for i, n in enumerate(names)}, **kw}
    return status(lib.molt_gated_scan_fwd(ctypes.byref(d), *[ptr[n] for n in names], FAKE, 16, None))


def scan_bwd(lib, d, **kw):
    names = ("dy", "gate", "value", "states", "h0", "cu", "dfinal", "dgate", "dvalue", "dinit")
    ptr = {**{n: FAKE * (i + 1) for i, n in enumerate(names)}, **kw}
    return status(lib.molt_gated_scan_bwd(ctypes.byref(d), *[ptr[n] for n in names], FAKE, 16, None))


def scan_step(lib, d, **kw):
    names = ("gate", "value", "state", "y", "out")
    ptr = {**{n: FAKE * (i + 1) for i, n in enumerate(names)}, **kw}
    return status(lib.molt_gated_scan_step(ctypes.byref(d), *[ptr[n] for n in names], None))


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), BAD), (dict(H=0), BAD), (dict(B=-1), BAD), (dict(dtype=3), BAD), (dict(form=2), BAD), (dict(form=-1), BAD),
    (dict(H=65537), SHAPE), (dict(T=(1 << 31) - 100), SHAPE), (dict(B=(1 << 31) - 1), SHAPE), (dict(gate_stride=63), BAD),
    (dict(value_stride=-1), BAD), (dict(dy_stride=1), BAD)])
def test_scan_refuses_descriptors(lib, kw, want):
    n0 = lib.molt_kernel_launches()
    assert scan_fwd(lib, scan(**kw)) == want
    assert scan_bwd(lib, scan(**kw)) == want
    assert scan_step(lib, scan(**{"T": 2, **kw})) == want
    assert lib.molt_kernel_launches() == n0


def test_scan_refuses_pointers(lib):
    for n in ("gate", "value", "y"):
        assert scan_fwd(lib, scan(), **{n: None}) == BAD, n
        assert scan_fwd(lib, scan(), **{n: FAKE + 1}) == BAD, n
    for n in ("h0", "cu", "final", "states"):
        assert scan_fwd(lib, scan(), **{n: FAKE + 2}) == BAD, n
    assert scan_fwd(lib, scan(T=5), cu=None) == BAD                       # no two equal sequences
    assert scan_fwd(lib, scan(T=5, B=0), cu=None) == BAD
    assert scan_fwd(lib, scan(T=0, B=0), gate=None) == "MOLT_OK"
    assert scan_fwd(lib, scan(T=0), gate=None, final=None) == "MOLT_OK"
    for n in ("dy", "gate", "value", "states", "dgate", "dvalue"):
        assert scan_bwd(lib, scan(), **{n: None}) == BAD, n
    for n in ("dy", "gate", "value", "dgate", "dvalue"):
        assert scan_bwd(lib, scan(), **{n: FAKE + 1}) == BAD, n
    for n in ("states", "h0", "dfinal", "dinit", "cu"):
        assert scan_bwd(lib, scan(), **{n: FAKE + 2}) == BAD, n
    assert scan_step(lib, scan()) == BAD                                  # T is not B
    for n in ("gate", "value", "state", "y", "out"):
        assert scan_step(lib, scan(T=2), **{n: None}) == BAD, n
        assert scan_step(lib, scan(T=2), **{n: FAKE + 1}) == BAD, n
    assert scan_step(lib, scan(T=0, B=0), gate=None) == "MOLT_OK"
    for f in (lib.molt_gated_scan_fwd, lib.molt_gated_scan_bwd, lib.molt_gated_scan_step):
        assert status(f(None, *[FAKE] * (len(f.argtypes) - 2), None)) == BAD
    assert scan_fwd(lib, scan()) == scan_bwd(lib, scan()) == "MOLT_ERR_WORKSPACE"
    assert lib.molt_gated_scan_workspace_bytes(ctypes.byref(scan())) > 0
    assert lib.molt_gated_scan_workspace_bytes(ctypes.byref(scan(H=0))) == 0


def dropout(lib, d, x=FAKE, r=None, words=None, out=2 * FAKE):
    return status(lib.molt_dropout(ctypes.byref(d), x, r, words, out, None))


@pytest.mark.parametrize("kw,want", [
    (dict(T=-1), BAD), (dict(H=0), BAD), (dict(H=65537), SHAPE), (dict(T=(1 << 32) + 1), SHAPE),
    (dict(first_row=(1 << 32) - 3), SHAPE), (dict(first_row=-1), SHAPE), (dict(p=-0.1), BAD), (dict(p=1.1), BAD),
    (dict(p=float("nan")), BAD), (dict(res_scale=float("inf")), BAD), (dict(dtype=3), BAD), (dict(out_dtype=1), BAD),
    (dict(x_stride=63), BAD), (dict(residual_stride=-64), BAD)])
def test_dropout_refuses_descriptors(lib, kw, want):
    n0 = lib.molt_kernel_launches()
    assert dropout(lib, drop(**kw)) == want
    assert lib.molt_kernel_launches() == n0


def test_dropout_refuses_pointers(lib):
    assert dropout(lib, drop(), x=None) == BAD
    assert dropout(lib, drop(), out=None) == BAD
    assert dropout(lib, drop(), x=FAKE + 1) == BAD
    assert dropout(lib, drop(out_dtype=2), out=FAKE + 2) == BAD
    assert dropout(lib, drop(), r=FAKE + 1) == BAD
    assert dropout(lib, drop(), words=FAKE + 4) == BAD
    assert dropout(lib, drop(out_dtype=2), out=FAKE) == BAD               # in place, another type
    assert dropout(lib, drop(x_stride=72), out=FAKE) == BAD               # in place, strided rows
    assert dropout(lib, drop(residual_stride=72), r=2 * FAKE) == BAD
    assert dropout(lib, drop(T=0), x=None, out=None) == "MOLT_OK"
    assert status(lib.molt_dropout(None, FAKE, None, None, FAKE, None)) == BAD


def test_outputs_that_share_memory_are_refused(lib):
    """... with another output, with the last byte of an input, or a strided input's."""
    n = 4 * 64 * 2   # bytes of four rows
    assert ffn_fwd(lib, ffn(), y=FAKE) == ffn_fwd(lib, ffn(), y=FAKE + n - 16) == ffn_fwd(lib, ffn(x_stride=128), y=FAKE + n) == BAD
    assert ffn_fwd(lib, ffn(), y=FAKE + n) == ffn_fwd(lib, ffn(x_stride=128), y=FAKE + 2 * n - 128) == "MOLT_ERR_WORKSPACE"
    assert ffn_fwd(lib, ffn(), gate_out=20 * FAKE, up_out=20 * FAKE + 1008) == BAD
    assert ffn_bwd(lib, ffn(), dx=FAKE) == ffn_bwd(lib, ffn(), dw_up=20 * FAKE, dw_gate=20 * FAKE) == BAD
    assert ffn_bwd(lib, ffn(), dw_up=20 * FAKE, dw_gate=20 * FAKE + 128 * 64 * 4) == "MOLT_ERR_WORKSPACE"
    assert scan_fwd(lib, scan(), y=FAKE) == scan_fwd(lib, scan(), final=3 * FAKE) == scan_fwd(lib, scan(gate_stride=128), y=FAKE + 800) == BAD
    assert scan_fwd(lib, scan(), final=3 * FAKE + 2 * 64 * 4) == "MOLT_ERR_WORKSPACE"
    assert scan_bwd(lib, scan(), dgate=FAKE) == scan_bwd(lib, scan(), dinit=5 * FAKE) == BAD
    assert scan_step(lib, scan(T=2), y=FAKE) == scan_step(lib, scan(T=2), out=3 * FAKE + 4) == scan_step(lib, scan(T=2), out=4 * FAKE) == BAD
    assert dropout(lib, drop(), out=FAKE + 16) == dropout(lib, drop(), r=3 * FAKE, out=3 * FAKE - 16) == BAD


def test_layouts_match_the_header(tmp_path):
    """The descriptors' sizes, and the constants, as a C compiler reads them."""
    import os
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "molt.h"\nint main(void) {\n'
                   '  printf("%zu %zu %zu %zu %zu %zu %d %d %d %d\\n", sizeof(molt_ffn_desc), offsetof(molt_ffn_desc, activation),\n'
                   '    sizeof(molt_scan_desc), offsetof(molt_scan_desc, fill_outside), sizeof(molt_dropout_desc),\n'
                   '    offsetof(molt_dropout_desc, out_dtype), MOLT_SCAN_STATE_ROWS, MOLT_ACT_GELU, MOLT_ACT_RELU, MOLT_SCAN_LOG);\n'
                   '  return 0;\n}\n')
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([gcc, "-std=c11", "-I", os.path.join(root, "include"), "-I", "/usr/local/cuda/include", str(src),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    vals = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert vals == [ctypes.sizeof(B.FfnDesc), B.FfnDesc.activation.offset, ctypes.sizeof(B.ScanDesc),
                    B.ScanDesc.fill_outside.offset, ctypes.sizeof(B.DropoutDesc), B.DropoutDesc.out_dtype.offset,
                    B.STATE_ROWS, B.ACTIVATIONS["gelu"], B.ACTIVATIONS["relu"], B.SCAN_FORMS["log"]]


def test_binding_refuses_host_tensors_and_wrong_shapes():
    bf = torch.bfloat16
    x, w, wd = torch.zeros(4, 64, dtype=bf), torch.zeros(128, 64, dtype=bf), torch.zeros(64, 128, dtype=bf)
    with pytest.raises(TypeError, match="CUDA"):
        molt.gated_ffn_fwd(x, w, w, wd)
    with pytest.raises(ValueError, match="w_up"):
        molt.gated_ffn_fwd(x, w, w[:64], wd)
    with pytest.raises(ValueError, match="w_down"):
        molt.gated_ffn_fwd(x, w, w, w)
    with pytest.raises(TypeError, match="float32"):
        molt.gated_ffn_fwd(x.float(), w.float(), w.float(), wd.float())
    with pytest.raises(ValueError, match="dy"):
        molt.gated_ffn_bwd(x[:2], x, w, w, wd)
    with pytest.raises(TypeError, match="CUDA"):
        molt.gated_scan_fwd(x, x)
    with pytest.raises(TypeError, match="CUDA"):
        molt.gated_scan_step(x, x, x.float())
    with pytest.raises(TypeError, match="CUDA"):
        molt.dropout_fwd(x, 0.1, 1)
    for f in (B._activation, B._form):
        with pytest.raises(ValueError, match="one of"):
            f("tanh")
