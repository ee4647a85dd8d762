"""The operators on the residual stream around the LM head: token embedding with
scaling and its gradient, and the norms after and before a block fused with its gate
and residual scale.  As in the rest of the binding, every function marshals its
arguments into the C ABI (include/molt.h) and runs on the current CUDA stream."""
from __future__ import annotations

import ctypes

from . import _check, _ptr, _stream, _torch, _workspace, load

_DTYPES = None


def _dtype_code(dtype, name):
    """molt_dtype of a torch type."""
    global _DTYPES
    if _DTYPES is None:
        torch = _torch()
        _DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be bfloat16, float16 or float32, got {dtype}")
    return code


def _shaped(t, shape, name):
    if tuple(t.shape) != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    return t


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the call's other tensors on {dev}")


def _rows(t, dtype, name):
    """(pointer, row stride) of a CUDA matrix whose rows are contiguous."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    T, H = t.shape
    if T <= 1 and (H <= 1 or t.stride(1) == 1):
        return t.data_ptr(), H
    if (H > 1 and t.stride(1) != 1) or t.stride(0) < H:
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), t.stride(0)


# ----------------------------------------------------------------- embedding
def token_embedding(weight, tokens, scale=1.0, out_dtype=None, out=None, stream=None):
    """scale * weight[tokens] as [T, H] of weight's type, or of `out_dtype` =
    float32 (molt_token_embedding).  A token outside [0, V) gives a row of zeros
    and sets the token-range bit of device_status()."""
    torch = _torch()
    V, H = weight.shape
    T, = tokens.shape
    dev = weight.device
    if out is None:
        out = torch.empty(T, H, dtype=weight.dtype if out_dtype is None else out_dtype, device=dev)
    else:
        _shaped(out, (T, H), "out")
    _same_device(dev, tokens=tokens, out=out)
    _check(load().molt_token_embedding(
        _ptr(weight, None, "weight"), _dtype_code(weight.dtype, "weight"), _ptr(tokens, torch.int32, "tokens"), T, H, V,
        float(scale), _ptr(out, out_dtype, "out"), _dtype_code(out.dtype, "out"), _stream(stream, dev.index)))
    return out


def token_embedding_bwd(dout, tokens, V, scale=1.0, padding_idx=None, dtype=None, dW=None, accumulate_dW=False,
                        stream=None, workspace=None):
    """The embedding's gradient, scale * the sum of dout's rows by token
    (molt_token_embedding_bwd), as [V, H] of dout's type, or of `dtype` = float32.
    With `dW` it is written there, with accumulate_dW (dW in float32: the head's
    gradient where the weights are tied) added.  Bitwise reproducible."""
    torch = _torch()
    T, H = dout.shape
    dev = dout.device
    _shaped(tokens, (T,), "tokens")
    if dW is None:
        dW = torch.empty(V, H, dtype=dout.dtype if dtype is None else dtype, device=dev)
        accumulate_dW = False
    else:
        _shaped(dW, (V, H), "dW")
    _same_device(dev, tokens=tokens, dW=dW)
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(int(L.molt_token_embedding_bwd_workspace_bytes(T, H, V)), dev, "embedding_bwd", stream)
    _check(L.molt_token_embedding_bwd(
        _ptr(dout, None, "dout"), _dtype_code(dout.dtype, "dout"), _ptr(tokens, torch.int32, "tokens"), T, H, V,
        float(scale), -1 if padding_idx is None else int(padding_idx), _ptr(dW, dtype, "dW"),
        _dtype_code(dW.dtype, "dW"), 1 if accumulate_dW else 0, ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return dW


# -------------------------------------------------------------- residual norm
class NormDesc(ctypes.Structure):
    """molt_norm_desc."""
    _fields_ = [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("residual_dtype", ctypes.c_int), ("param_dtype", ctypes.c_int), ("gate_kind", ctypes.c_int),
                ("res_scale", ctypes.c_float), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float)]


GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = range(4)


def _gate_kind(gate, T, H):
    """The gate's kind by its shape: [H], [T, 1] or [T] (where T is not H; then [T, 1] is needed), [T, H]."""
    if gate is None:
        return GATE_NONE
    shape = tuple(gate.shape)
    if shape == (H,):
        return GATE_CHANNEL
    if shape in ((T,), (T, 1)):
        return GATE_TOKEN
    if shape == (T, H):
        return GATE_FULL
    raise ValueError(f"gate must have shape [{H}], [{T}], [{T}, 1] or [{T}, {H}], got {list(shape)}")


def _params(dtype, H, **named):
    """The common type of the parameter vectors (x's where there is none)."""
    torch = _torch()
    found = None
    for name, p in named.items():
        if p is None:
            continue
        _shaped(p, (H,), name)
        if p.dtype not in (dtype, torch.float32):
            raise TypeError(f"{name} must be {dtype} or float32, got {p.dtype}")
        if found not in (None, p.dtype):
            raise TypeError("w_post, w_pre and a channel gate must have one type")
        found = p.dtype
    return dtype if found is None else found


def residual_norm_fwd(x, residual=None, w_post=None, gate=None, w_pre=None, res_scale=1.0, eps=1e-6, weight_offset=0.0,
                      residual_dtype=None, want_stats=True, stream=None):
    """A block's output x into the residual stream, and out of it again
    (molt_residual_norm_fwd):
        u = x, or RMS norm of x with weight w_post;  r' = res_scale residual + gate u;
        y = RMS norm of r' with weight w_pre.
    x, residual [T, H] (rows may be strided); gate [H], [T, 1] (fp32), [T, H] or None;
    w_post, w_pre [H] or None.  residual_dtype (without a residual: x's type or
    float32) is the stream's type.  Returns dict(y, residual = r', rstd_post,
    rstd_pre); what a call has no use for is None, and r' is x itself where nothing
    changes it (no residual, norm or gate)."""
    torch = _torch()
    T, H = x.shape
    dev, dtype = x.device, x.dtype
    kind = _gate_kind(gate, T, H)
    if residual is not None:
        _shaped(residual, (T, H), "residual")
        if residual_dtype not in (None, residual.dtype):
            raise TypeError("residual_dtype is the residual's own type")
        residual_dtype = residual.dtype
    elif residual_dtype is None:
        residual_dtype = dtype
    same = residual is None and w_post is None and kind == GATE_NONE and residual_dtype == dtype
    ptype = _params(dtype, H, w_post=w_post, w_pre=w_pre, gate=gate if kind == GATE_CHANNEL else None)
    _same_device(dev, residual=residual, w_post=w_post, gate=gate, w_pre=w_pre)
    f32 = torch.float32
    out = {"y": torch.empty(T, H, dtype=dtype, device=dev) if w_pre is not None else None,
           "residual": x if same else torch.empty(T, H, dtype=residual_dtype, device=dev),
           "rstd_post": torch.empty(T, dtype=f32, device=dev) if want_stats and w_post is not None else None,
           "rstd_pre": torch.empty(T, dtype=f32, device=dev) if want_stats and w_pre is not None else None}
    if same and w_pre is None:
        return out
    xp, xs = _rows(x, dtype, "x")
    rp, rs = _rows(residual, residual_dtype, "residual")
    desc = NormDesc(T, H, xs, rs, 0, _dtype_code(dtype, "x"), _dtype_code(residual_dtype, "residual"),
                    _dtype_code(ptype, "w_pre"), kind, float(res_scale), float(eps), float(weight_offset))
    _check(load().molt_residual_norm_fwd(
        ctypes.byref(desc), xp, rp, _ptr(w_post, None, "w_post"),
        _ptr(gate, f32 if kind == GATE_TOKEN else dtype if kind == GATE_FULL else None, "gate"),
        _ptr(w_pre, None, "w_pre"), _ptr(out["y"]), None if same else _ptr(out["residual"]), _ptr(out["rstd_post"]),
        _ptr(out["rstd_pre"]), _stream(stream, dev.index)))
    return out


def residual_norm_bwd(dy, dresidual, x, residual, rstd_pre, rstd_post=None, w_post=None, gate=None, w_pre=None,
                      res_scale=1.0, weight_offset=0.0, want_dresidual=True, dw_post=None, dgate=None, dw_pre=None,
                      accumulate=False, stream=None, workspace=None):
    """Gradients of residual_norm_fwd (molt_residual_norm_bwd) from dy (the gradient
    of y, None without w_pre) and dresidual (that of r' from later blocks, or None).
    x, gate and weights as there; residual is its r', rstd_* its statistics.  Returns
    dict(dx, dresidual, dw_post, dgate, dw_pre): weights' gradients fp32 [H], the
    gate's fp32 [H] or [T], or [T, H] of x's type.  Buffers given for dw_post, dw_pre
    and a channel gate's dgate are written, with accumulate=True added to."""
    torch = _torch()
    T, H = x.shape
    dev, dtype, f32 = x.device, x.dtype, torch.float32
    kind = _gate_kind(gate, T, H)
    if residual is None and dresidual is None:
        raise ValueError("one of residual and dresidual is needed")
    rtype = (residual if residual is not None else dresidual).dtype
    for name, t in (("dy", dy), ("dresidual", dresidual), ("residual", residual)):
        if t is not None:
            _shaped(t, (T, H), name)
    for name, t in (("rstd_pre", rstd_pre), ("rstd_post", rstd_post)):
        if t is not None:
            _shaped(t, (T,), name)
    ptype = _params(dtype, H, w_post=w_post, w_pre=w_pre, gate=gate if kind == GATE_CHANNEL else None)
    _same_device(dev, dy=dy, dresidual=dresidual, residual=residual, rstd_pre=rstd_pre, rstd_post=rstd_post,
                 w_post=w_post, gate=gate, w_pre=w_pre, dw_post=dw_post, dgate=dgate, dw_pre=dw_pre)

    def vector(given, wanted, name):
        if not wanted:
            return None
        if given is None:
            return (torch.zeros if accumulate else torch.empty)(H, dtype=f32, device=dev)
        return _shaped(given, (H,), name)

    if dgate is not None and kind != GATE_CHANNEL:
        raise ValueError("dgate can be given for a channel gate only")
    out = {"dx": torch.empty(T, H, dtype=dtype, device=dev),
           "dresidual": torch.empty(T, H, dtype=rtype, device=dev) if want_dresidual else None,
           "dw_post": vector(dw_post, w_post is not None, "dw_post"),
           "dgate": vector(dgate, kind == GATE_CHANNEL, "dgate"),
           "dw_pre": vector(dw_pre, w_pre is not None, "dw_pre")}
    if kind == GATE_TOKEN:
        out["dgate"] = torch.empty(T, dtype=f32, device=dev)
    elif kind == GATE_FULL:
        out["dgate"] = torch.empty(T, H, dtype=dtype, device=dev)
    xp, xs = _rows(x, dtype, "x")
    rp, rs = _rows(residual, rtype, "residual")
    dyp, dys = _rows(dy, dtype, "dy")
    desc = NormDesc(T, H, xs, rs, dys, _dtype_code(dtype, "x"), _dtype_code(rtype, "residual"),
                    _dtype_code(ptype, "w_pre"), kind, float(res_scale), 0.0, float(weight_offset))
    ref = ctypes.byref(desc)
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(int(L.molt_residual_norm_bwd_workspace_bytes(ref)), dev, "norm_bwd", stream)
    _check(L.molt_residual_norm_bwd(
        ref, dyp, _ptr(dresidual, rtype, "dresidual"), xp, rp, _ptr(rstd_post, f32, "rstd_post"),
        _ptr(rstd_pre, f32, "rstd_pre"), _ptr(w_post, None, "w_post"),
        _ptr(gate, f32 if kind == GATE_TOKEN else dtype if kind == GATE_FULL else None, "gate"),
        _ptr(w_pre, None, "w_pre"), _ptr(out["dx"]), _ptr(out["dresidual"]), _ptr(out["dw_post"], f32, "dw_post"),
        _ptr(out["dgate"], dtype if kind == GATE_FULL else f32, "dgate"), _ptr(out["dw_pre"], f32, "dw_pre"),
        1 if accumulate else 0, ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return out
