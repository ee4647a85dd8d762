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
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {list(shape)}, got {list(t.shape)}")
    return t


def _same_device(dev, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != dev:
            raise ValueError(f"{name} is on {t.device}, the call's other tensors on {dev}")


def _cuda(t, name):
    """The CUDA device of a tensor."""
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.device


def _at(t, dtype, dev, name):
    """Pointer of a contiguous tensor of this type on this device (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is not dtype or t.device != dev or not t.is_contiguous():
        _same_device(dev, **{name: t})
        return _ptr(t, dtype, name)
    return t.data_ptr()


def _rows(t, dtype, dev, name):
    """(pointer, row stride, 0 for rows side by side) of a matrix whose rows are contiguous."""
    if t is None:
        return None, 0
    if t.is_contiguous():
        return _at(t, dtype, dev, name), 0
    _same_device(dev, **{name: t})
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    T, H = t.shape
    if (H > 1 and t.stride(1) != 1) or (T > 1 and t.stride(0) < H):
        raise ValueError(f"{name} must have contiguous rows that do not overlap")
    return t.data_ptr(), t.stride(0) if T > 1 else 0


# ----------------------------------------------------------------- embedding
def token_embedding(weight, tokens, scale=1.0, out_dtype=None, out=None, stream=None):
    """scale * weight[tokens] as [T, H] of weight's type, or of `out_dtype` =
    float32 (molt_token_embedding).  A token outside [0, V) gives a row of zeros
    and sets the token-range bit of device_status()."""
    torch = _torch()
    V, H = weight.shape
    T, = tokens.shape
    dev, dtype = _cuda(weight, "weight"), weight.dtype
    if out is None:
        out = torch.empty(T, H, dtype=dtype if out_dtype is None else out_dtype, device=dev)
    else:
        _shaped(out, (T, H), "out")
    _check(load().molt_token_embedding(
        _at(weight, dtype, dev, "weight"), _dtype_code(dtype, "weight"), _at(tokens, torch.int32, dev, "tokens"), T, H,
        V, scale, _at(out, out_dtype or out.dtype, dev, "out"), _dtype_code(out.dtype, "out"),
        _stream(stream, dev.index)))
    return out


def token_embedding_bwd(dout, tokens, V, scale=1.0, padding_idx=None, dtype=None, dW=None, accumulate_dW=False,
                        stream=None, workspace=None):
    """The embedding's gradient, scale * the sum of dout's rows by token
    (molt_token_embedding_bwd), as [V, H] of dout's type, or of `dtype` = float32.
    With `dW` it is written there, with accumulate_dW (dW in float32: the head's
    gradient where the weights are tied) added.  Bitwise reproducible."""
    torch = _torch()
    T, H = dout.shape
    _shaped(tokens, (T,), "tokens")
    dev, din = _cuda(dout, "dout"), dout.dtype
    if dW is None:
        dW = torch.empty(V, H, dtype=din if dtype is None else dtype, device=dev)
        accumulate_dW = False
    else:
        _shaped(dW, (V, H), "dW")
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(L.molt_token_embedding_bwd_workspace_bytes(T, H, V), dev, "embedding_bwd", stream)
    _check(L.molt_token_embedding_bwd(
        _at(dout, din, dev, "dout"), _dtype_code(din, "dout"), _at(tokens, torch.int32, dev, "tokens"), T, H, V, scale,
        -1 if padding_idx is None else padding_idx, _at(dW, dtype or dW.dtype, dev, "dW"), _dtype_code(dW.dtype, "dW"),
        1 if accumulate_dW else 0, ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return dW


# -------------------------------------------------------------- residual norm
class NormDesc(ctypes.Structure):
    """molt_norm_desc."""
    _fields_ = [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("dy_stride", ctypes.c_int64), ("dtype", ctypes.c_int),
                ("residual_dtype", ctypes.c_int), ("param_dtype", ctypes.c_int), ("gate_kind", ctypes.c_int),
                ("res_scale", ctypes.c_float), ("eps", ctypes.c_float), ("weight_offset", ctypes.c_float)]


GATE_NONE, GATE_CHANNEL, GATE_TOKEN, GATE_FULL = range(4)

# Descriptors by their values, with the backward's workspace bytes: building one takes
# longer than the rest of a small call's marshalling.  They are read only.
_desc_cache: dict = {}
_DESC_CACHE_MAX = 256


def _desc(device, *values):
    """Reference to the molt_norm_desc of these values, and its backward's workspace bytes."""
    key = (device, values)
    entry = _desc_cache.get(key)
    if entry is None:
        if len(_desc_cache) >= _DESC_CACHE_MAX:
            _desc_cache.clear()
        ref = ctypes.byref(NormDesc(*values))
        entry = _desc_cache[key] = ref, load().molt_residual_norm_bwd_workspace_bytes(ref)
    return entry


_KINDS = {"channel": GATE_CHANNEL, "token": GATE_TOKEN, "full": GATE_FULL}


def _gate_kind(gate, T, H, stated=None):
    """The gate's kind, by its shape or as stated: [H], [T, 1] or [T], [T, H].  A float32 vector
    of T = H could be a gate per channel or per token: its kind has to be stated."""
    if gate is None:
        if stated is not None:
            raise ValueError(f"gate_kind is {stated!r}, but there is no gate")
        return GATE_NONE
    shape = gate.shape
    if stated is not None:
        shapes = {"channel": ((H,),), "token": ((T, 1), (T,)), "full": ((T, H),)}.get(stated, ())
        if shape not in shapes:
            raise ValueError(f"a gate of shape {list(shape)} is not of kind {stated!r} (channel [{H}], token [{T}, 1], full [{T}, {H}])")
        return _KINDS[stated]
    if shape == (H,):
        if T == H > 1 and gate.dtype is _torch().float32:
            raise ValueError(f"a gate of shape [{H}] with {T} rows could be of a channel or of a token: state its "
                             "gate_kind, or give a token's as [T, 1]")
        return GATE_CHANNEL
    if shape == (T,) or shape == (T, 1):
        return GATE_TOKEN
    if shape == (T, H):
        return GATE_FULL
    raise ValueError(f"gate must have shape [{H}], [{T}], [{T}, 1] or [{T}, {H}], got {list(shape)}")


def _param_type(dtype, H, w_post, w_pre, gate):
    """The common type of the parameter vectors (x's where there is none)."""
    found = None
    for name, p in (("w_post", w_post), ("w_pre", w_pre), ("gate", gate)):
        if p is None:
            continue
        _shaped(p, (H,), name)
        t = p.dtype
        if t is not dtype and t is not _torch().float32:
            raise TypeError(f"{name} must be {dtype} or float32, got {t}")
        if found is not None and found is not t:
            raise TypeError("w_post, w_pre and a channel gate must have one type")
        found = t
    return dtype if found is None else found


def residual_norm_fwd(x, residual=None, w_post=None, gate=None, w_pre=None, res_scale=1.0, eps=1e-6, weight_offset=0.0,
                      residual_dtype=None, want_stats=True, stream=None, gate_kind=None):
    """A block's output x into the residual stream, and out of it again
    (molt_residual_norm_fwd):
        u = x, or RMS norm of x with weight w_post;  r' = res_scale residual + gate u;
        y = RMS norm of r' with weight w_pre.
    x, residual [T, H] (rows may be strided); w_post, w_pre [H] or None; gate [H], [T, 1] or
    [T] (fp32), [T, H] or None.  gate_kind = "channel", "token" or "full" states what the
    gate is; a float32 vector needs it where T = H, and a program whose T changes gives it
    always.  residual_dtype (without a residual: x's type or float32) is the stream's
    type.  Returns dict(y, residual = r', rstd_post, rstd_pre); what a call has no use for
    is None, and r' is x itself where nothing changes it (no residual, norm or gate)."""
    torch = _torch()
    T, H = x.shape
    kind = _gate_kind(gate, T, H, gate_kind)
    dtype, f32 = x.dtype, torch.float32
    if residual is not None:
        _shaped(residual, (T, H), "residual")
        rtype = residual.dtype
        if residual_dtype is not None and residual_dtype is not rtype:
            raise TypeError("residual_dtype is the residual's own type")
    else:
        rtype = dtype if residual_dtype is None else residual_dtype
    ptype = _param_type(dtype, H, w_post, w_pre, gate if kind == GATE_CHANNEL else None)
    dev = _cuda(x, "x")
    same = residual is None and w_post is None and kind == GATE_NONE and rtype is dtype
    xp, xs = _rows(x, dtype, dev, "x")
    rp, rs = _rows(residual, rtype, dev, "residual")
    y = torch.empty(T, H, dtype=dtype, device=dev) if w_pre is not None else None
    r_out = x if same else torch.empty(T, H, dtype=rtype, device=dev)
    rstd_post = torch.empty(T, dtype=f32, device=dev) if want_stats and w_post is not None else None
    rstd_pre = torch.empty(T, dtype=f32, device=dev) if want_stats and w_pre is not None else None
    out = {"y": y, "residual": r_out, "rstd_post": rstd_post, "rstd_pre": rstd_pre}
    if same and y is None:
        return out
    ref, _ = _desc(dev, T, H, xs, rs, 0, _dtype_code(dtype, "x"), _dtype_code(rtype, "residual"),
                   _dtype_code(ptype, "w_pre"), kind, res_scale, eps, weight_offset)
    _check(load().molt_residual_norm_fwd(
        ref, xp, rp, _at(w_post, ptype, dev, "w_post"),
        _at(gate, ptype if kind == GATE_CHANNEL else f32 if kind == GATE_TOKEN else dtype, dev, "gate"),
        _at(w_pre, ptype, dev, "w_pre"), y if y is None else y.data_ptr(), None if same else r_out.data_ptr(),
        rstd_post if rstd_post is None else rstd_post.data_ptr(), rstd_pre if rstd_pre is None else rstd_pre.data_ptr(),
        _stream(stream, dev.index)))
    return out


def residual_norm_bwd(dy, dresidual, x, residual, rstd_pre, rstd_post=None, w_post=None, gate=None, w_pre=None,
                      res_scale=1.0, weight_offset=0.0, want_dresidual=True, dw_post=None, dgate=None, dw_pre=None,
                      accumulate=False, stream=None, workspace=None, gate_kind=None):
    """Gradients of residual_norm_fwd (molt_residual_norm_bwd) from dy (the gradient
    of y, None without w_pre) and dresidual (that of r' from later blocks, or None).
    x, gate, gate_kind and weights as there; residual is its r', rstd_* its statistics.  Returns
    dict(dx, dresidual, dw_post, dgate, dw_pre): weights' gradients fp32 [H], the
    gate's fp32 [H] or [T], or [T, H] of x's type.  Buffers given for dw_post, dw_pre
    and a channel gate's dgate are written, with accumulate=True added to."""
    torch = _torch()
    T, H = x.shape
    dtype, f32 = x.dtype, torch.float32
    kind = _gate_kind(gate, T, H, gate_kind)
    if residual is None and dresidual is None:
        raise ValueError("one of residual and dresidual is needed")
    rtype = (residual if residual is not None else dresidual).dtype
    for name, t in (("dy", dy), ("dresidual", dresidual), ("residual", residual)):
        if t is not None:
            _shaped(t, (T, H), name)
    for name, t in (("rstd_pre", rstd_pre), ("rstd_post", rstd_post)):
        if t is not None:
            _shaped(t, (T,), name)
    ptype = _param_type(dtype, H, w_post, w_pre, gate if kind == GATE_CHANNEL else None)
    dev = _cuda(x, "x")

    def vector(given, wanted, name):
        if not wanted:
            return None
        if given is None:
            return (torch.zeros if accumulate else torch.empty)(H, dtype=f32, device=dev)
        return _shaped(given, (H,), name)

    if dgate is not None and kind != GATE_CHANNEL:
        raise ValueError("dgate can be given for a channel gate only")
    dx = torch.empty(T, H, dtype=dtype, device=dev)
    dr_out = torch.empty(T, H, dtype=rtype, device=dev) if want_dresidual else None
    dw_post = vector(dw_post, w_post is not None, "dw_post")
    dw_pre = vector(dw_pre, w_pre is not None, "dw_pre")
    if kind == GATE_TOKEN:
        dgate = torch.empty(T, dtype=f32, device=dev)
    elif kind == GATE_FULL:
        dgate = torch.empty(T, H, dtype=dtype, device=dev)
    else:
        dgate = vector(dgate, kind == GATE_CHANNEL, "dgate")
    xp, xs = _rows(x, dtype, dev, "x")
    rp, rs = _rows(residual, rtype, dev, "residual")
    dyp, dys = _rows(dy, dtype, dev, "dy")
    ref, nbytes = _desc(dev, T, H, xs, rs, dys, _dtype_code(dtype, "x"), _dtype_code(rtype, "residual"),
                        _dtype_code(ptype, "w_pre"), kind, res_scale, 0.0, weight_offset)
    ws = workspace
    if ws is None:
        ws = _workspace(nbytes, dev, "norm_bwd", stream)
    _check(load().molt_residual_norm_bwd(
        ref, dyp, _at(dresidual, rtype, dev, "dresidual"), xp, rp, _at(rstd_post, f32, dev, "rstd_post"),
        _at(rstd_pre, f32, dev, "rstd_pre"), _at(w_post, ptype, dev, "w_post"),
        _at(gate, ptype if kind == GATE_CHANNEL else f32 if kind == GATE_TOKEN else dtype, dev, "gate"),
        _at(w_pre, ptype, dev, "w_pre"), dx.data_ptr(), dr_out if dr_out is None else dr_out.data_ptr(),
        _at(dw_post, f32, dev, "dw_post"), _at(dgate, dtype if kind == GATE_FULL else f32, dev, "dgate"),
        _at(dw_pre, f32, dev, "dw_pre"), 1 if accumulate else 0, ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return {"dx": dx, "dresidual": dr_out, "dw_post": dw_post, "dgate": dgate, "dw_pre": dw_pre}
