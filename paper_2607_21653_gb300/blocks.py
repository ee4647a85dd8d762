"""The operators inside a block, between two norms of the residual stream: the gated
feed-forward block, the gated linear recurrence over packed sequences and dropout from a
counter, with their gradients.  As in the rest of the binding, every function marshals its
arguments into the C ABI (include/molt.h) and runs on the current CUDA stream of its
tensors' device, or on `stream`; what it returns belongs to that stream."""
from __future__ import annotations

import ctypes

from . import _check, _on_stream, _stream, _torch, _workspace, load
from .stream import _at, _cuda, _dtype_code, _rows, _shaped

ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}
SCAN_FORMS = {"sigmoid": 0, "log": 1}
STATE_ROWS = 128      # MOLT_SCAN_STATE_ROWS


class FfnDesc(ctypes.Structure):
    """molt_ffn_desc."""
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "H", "F", "x_stride", "w_gate_stride", "w_up_stride", "w_down_stride",
                                               "dy_stride")] + [("dtype", ctypes.c_int), ("activation", ctypes.c_int)]


class ScanDesc(ctypes.Structure):
    """molt_scan_desc."""
    _fields_ = [(n, ctypes.c_int64) for n in ("T", "H", "B", "gate_stride", "value_stride", "dy_stride")] + [
        (n, ctypes.c_int) for n in ("dtype", "form", "fill_outside")]


class DropoutDesc(ctypes.Structure):
    """molt_dropout_desc."""
    _fields_ = [("T", ctypes.c_int64), ("H", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("residual_stride", ctypes.c_int64), ("first_row", ctypes.c_int64), ("seed", ctypes.c_uint64),
                ("offset", ctypes.c_uint64), ("p", ctypes.c_double), ("res_scale", ctypes.c_float),
                ("dtype", ctypes.c_int), ("out_dtype", ctypes.c_int)]


def _call(fn, dev, *args):
    """A call of the C ABI with the tensors' device as the current one."""
    torch = _torch()
    if torch._C._cuda_getDevice() == dev.index:
        status = fn(*args)
        if status:
            _check(status)
        return
    with torch.cuda.device(dev):
        _check(fn(*args))


def _handle(stream, dev):
    """cudaStream_t of a call on tensors of this device."""
    if stream is not None and stream.device != dev:
        raise ValueError(f"stream is on {stream.device}, the call's tensors on {dev}")
    return _stream(stream, dev.index)


# The checks of _at and _rows (.stream) in the order in which a good argument passes soonest: the
# marshalling of a small call takes longer than its kernels.
def _vec(t, dtype, dev, name):
    """Pointer of a contiguous tensor of this type on this device (None -> NULL)."""
    if t is None:
        return None
    if t.dtype is dtype and t.is_contiguous() and t.get_device() == dev.index:
        return t.data_ptr()
    return _at(t, dtype, dev, name)


def _mat(t, dtype, dev, name):
    """(pointer, row stride, 0 for rows side by side) of a matrix whose rows are contiguous."""
    if t is not None and t.dtype is dtype and t.is_contiguous() and t.get_device() == dev.index:
        return t.data_ptr(), 0
    return _rows(t, dtype, dev, name)


def _scratch(nbytes, dev, key, stream):
    """Workspace of a call: the binding's buffer of this stream, or inside a capture memory of
    the graph's own pool (a buffer that other calls share could be replaced under the graph)."""
    torch = _torch()
    if not torch._C._cuda_isCurrentStreamCapturing():
        return _workspace(nbytes, dev, key, stream)
    with torch.cuda.stream(torch.cuda.current_stream(dev) if stream is None else stream):
        return torch.empty(nbytes, dtype=torch.uint8, device=dev)


# Descriptors by their values, with the workspace bytes of the call, by device: read only.
_desc_cache: dict = {}
_DESC_CACHE_MAX = 256


def _desc(dev, cls, values, query=None, *more):
    key = (dev.index, cls, values, query, more)
    entry = _desc_cache.get(key)
    if entry is None:
        if len(_desc_cache) >= _DESC_CACHE_MAX:
            _desc_cache.clear()
        ref, nbytes = ctypes.byref(cls(*values)), 0
        if query:
            with _torch().cuda.device(dev):   # a size can go by the device's SMs
                nbytes = getattr(load(), query)(ref, *more)
        entry = _desc_cache[key] = ref, nbytes
    return entry


# --------------------------------------------------------- gated feed-forward
def _activation(name):
    code = ACTIVATIONS.get(name)
    if code is None:
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, got {name!r}")
    return code


def _ffn_shapes(x, w_gate, w_up, w_down):
    T, H = x.shape
    F = w_gate.shape[0]
    _shaped(w_gate, (F, H), "w_gate")
    _shaped(w_up, (F, H), "w_up")
    _shaped(w_down, (H, F), "w_down")
    if x.dtype is _torch().float32:
        raise TypeError("the feed-forward block is computed on bfloat16 or float16, got float32")
    return T, H, F


@_on_stream
def gated_ffn_fwd(x, w_gate, w_up, w_down, activation="silu", keep=False, stream=None, workspace=None):
    """Gated feed-forward block (molt_gated_ffn_fwd):
        y = (act(x w_gate^T) * (x w_up^T)) w_down^T
    x [T, H], w_gate and w_up [F, H], w_down [H, F], bfloat16 or float16, H and F multiples of
    8, rows may be strided by multiples of 8; act(..) * (..) is rounded to x's type before the second
    product (in float16 it is infinite past 65504).  activation: "silu", "gelu" (its tanh form),
    "relu".  Returns dict(y [T, H], gate, up): with keep=True the two products [T, F] for
    the backward, else None."""
    torch = _torch()
    T, H, F = _ffn_shapes(x, w_gate, w_up, w_down)
    dev, dtype = _cuda(x, "x"), x.dtype
    xp, xs = _mat(x, dtype, dev, "x")
    gp, gs = _mat(w_gate, dtype, dev, "w_gate")
    up, us = _mat(w_up, dtype, dev, "w_up")
    dp, ds = _mat(w_down, dtype, dev, "w_down")
    y = torch.empty(T, H, dtype=dtype, device=dev)
    gate = torch.empty(T, F, dtype=dtype, device=dev) if keep else None
    upo = torch.empty(T, F, dtype=dtype, device=dev) if keep else None
    ref, nbytes = _desc(dev, FfnDesc, (T, H, F, xs, gs, us, ds, 0, _dtype_code(dtype, "x"), _activation(activation)),
                        "molt_gated_ffn_fwd_workspace_bytes")
    ws = workspace if workspace is not None else _scratch(nbytes, dev, "gated_ffn", stream)
    _call(load().molt_gated_ffn_fwd, dev, ref, xp, gp, up, dp, y.data_ptr(), gate if gate is None else gate.data_ptr(),
          upo if upo is None else upo.data_ptr(), ws.data_ptr(), ws.numel(), _handle(stream, dev))
    return {"y": y, "gate": gate, "up": upo}


@_on_stream
def gated_ffn_bwd(dy, x, w_gate, w_up, w_down, gate=None, up=None, activation="silu", dw_dtype=None, dw_gate=None,
                  dw_up=None, dw_down=None, accumulate=False, stream=None, workspace=None):
    """Gradients of gated_ffn_fwd (molt_gated_ffn_bwd) from dy [T, H].  gate, up: what the
    forward kept; without them the two products are formed again.  Returns dict(dx, dw_gate,
    dw_up, dw_down), the weights' gradients in float32, or `dw_dtype` = x's type.  Buffers
    given for them (float32 or x's type, all three) are written, with accumulate=True (float32)
    added to."""
    torch = _torch()
    T, H, F = _ffn_shapes(x, w_gate, w_up, w_down)
    _shaped(dy, (T, H), "dy")
    dev, dtype = _cuda(x, "x"), x.dtype
    given = (dw_gate, dw_up, dw_down)
    shapes = (("dw_gate", (F, H)), ("dw_up", (F, H)), ("dw_down", (H, F)))
    if any(t is not None for t in given):
        if any(t is None for t in given):
            raise ValueError("buffers are given for all three weights' gradients or for none")
        if dw_dtype is not None and dw_dtype is not given[0].dtype:
            raise TypeError("dw_dtype is the buffers' own type")
        dw_dtype = given[0].dtype
        for t, (name, shape) in zip(given, shapes):
            _shaped(t, shape, name)
    else:
        dw_dtype = torch.float32 if dw_dtype is None else dw_dtype
        make = torch.zeros if accumulate else torch.empty
        given = tuple(make(*shape, dtype=dw_dtype, device=dev) for _, shape in shapes)
    for t, name in ((gate, "gate"), (up, "up")):
        if t is not None:
            _shaped(t, (T, F), name)
    if (gate is None) != (up is None):
        raise ValueError("gate and up come together")
    dyp, dys = _mat(dy, dtype, dev, "dy")
    xp, xs = _mat(x, dtype, dev, "x")
    gp, gs = _mat(w_gate, dtype, dev, "w_gate")
    upp, us = _mat(w_up, dtype, dev, "w_up")
    dp, ds = _mat(w_down, dtype, dev, "w_down")
    dx = torch.empty(T, H, dtype=dtype, device=dev)
    ref, nbytes = _desc(dev, FfnDesc, (T, H, F, xs, gs, us, ds, dys, _dtype_code(dtype, "x"), _activation(activation)),
                        "molt_gated_ffn_bwd_workspace_bytes", 0 if gate is None else 1)
    ws = workspace if workspace is not None else _scratch(nbytes, dev, "gated_ffn", stream)
    _call(load().molt_gated_ffn_bwd, dev, ref, dyp, xp, gp, upp, dp, _vec(gate, dtype, dev, "gate"), _vec(up, dtype, dev, "up"),
          dx.data_ptr(), *[_vec(t, dw_dtype, dev, name) for t, (name, _) in zip(given, shapes)],
          _dtype_code(dw_dtype, "dw_dtype"), 1 if accumulate else 0, ws.data_ptr(), ws.numel(), _handle(stream, dev))
    return {"dx": dx, "dw_gate": given[0], "dw_up": given[1], "dw_down": given[2]}


# ------------------------------------------------------- gated linear recurrence
def _form(kind):
    code = SCAN_FORMS.get(kind)
    if code is None:
        raise ValueError(f"kind must be one of {sorted(SCAN_FORMS)}, got {kind!r}")
    return code


def _scan_shapes(gate, cu_seqlens, dev):
    """(T, H, B, pointer of cu_seqlens) of packed rows [T, H] or equal sequences [B, L, H]."""
    if gate.dim() == 3:
        if cu_seqlens is not None:
            raise ValueError("cu_seqlens goes with packed rows [T, H]")
        B, L, H = gate.shape
        return B * L, H, B, None
    T, H = gate.shape
    if cu_seqlens is None:
        return T, H, 1, None
    n, = cu_seqlens.shape
    if n < 1:
        raise ValueError("cu_seqlens has one entry more than there are sequences")
    return T, H, n - 1, _vec(cu_seqlens, _torch().int32, dev, "cu_seqlens")


def _packed(t, like, name):
    """A [B, L, H] tensor as [B L, H]: rows evenly spaced."""
    _shaped(t, like.shape, name)
    return t if t.dim() == 2 else t.view(-1, t.shape[2])


@_on_stream
def gated_scan_fwd(gate, value, initial_state=None, cu_seqlens=None, kind="sigmoid", want_states=False,
                   want_final_state=True, out=None, stream=None, workspace=None):
    """Gated linear recurrence over sequences, channel by channel (molt_gated_scan_fwd):
        "sigmoid":  h_t = a_t h_{t-1} + (1 - a_t) value_t,  a_t = sigmoid(gate_t)
        "log":      h_t = a_t h_{t-1} + value_t,            a_t = exp(gate_t)
    (gates of the log form are at most 0, or the product of a sequence's a_t stays in float32's
    range).  gate, value: packed rows [T, H] of the sequences cu_seqlens [B + 1] (int32, on the device;
    None: one sequence), or [B, L, H]; bfloat16, float16 or float32, rows may be strided.
    initial_state [B, H] float32 or None.  Returns dict(y = h, final_state [B, H] float32, states):
    with want_states=True what the backward reads, else None.  Rows of a given `out` outside of
    every sequence stay as they were; without `out` they are 0."""
    torch = _torch()
    dev, dtype = _cuda(gate, "gate"), gate.dtype
    T, H, B, cu = _scan_shapes(gate, cu_seqlens, dev)
    gp, gs = _mat(_packed(gate, gate, "gate"), dtype, dev, "gate")
    vp, vs = _mat(_packed(value, gate, "value"), dtype, dev, "value")
    f32 = torch.float32
    if initial_state is not None:
        _shaped(initial_state, (B, H), "initial_state")
    fill = 1 if out is None else 0
    if out is None:
        out = torch.empty(gate.shape, dtype=dtype, device=dev)
    final = torch.empty(B, H, dtype=f32, device=dev) if want_final_state else None
    states = torch.empty((T + STATE_ROWS - 1) // STATE_ROWS, H, dtype=f32, device=dev) if want_states else None
    ref, nbytes = _desc(dev, ScanDesc, (T, H, B, gs, vs, 0, _dtype_code(dtype, "gate"), _form(kind), fill),
                        "molt_gated_scan_workspace_bytes")
    ws = workspace if workspace is not None else _scratch(nbytes, dev, "gated_scan", stream)
    _call(load().molt_gated_scan_fwd, dev, ref, gp, vp, _vec(initial_state, f32, dev, "initial_state"), cu,
          _vec(_shaped(out, gate.shape, "out"), dtype, dev, "out"), final if final is None else final.data_ptr(),
          states if states is None else states.data_ptr(), ws.data_ptr(), ws.numel(), _handle(stream, dev))
    return {"y": out, "final_state": final, "states": states}


@_on_stream
def gated_scan_bwd(dy, gate, value, states, initial_state=None, cu_seqlens=None, dfinal_state=None, kind="sigmoid",
                   stream=None, workspace=None):
    """Gradients of gated_scan_fwd (molt_gated_scan_bwd) from dy and dfinal_state [B, H]
    (float32, or None: the final state is not used), with the forward's inputs and its `states`.
    Returns dict(dgate, dvalue, dinitial_state), the last one None without an initial state.
    Rows outside of every sequence have gradients of 0."""
    torch = _torch()
    dev, dtype = _cuda(gate, "gate"), gate.dtype
    T, H, B, cu = _scan_shapes(gate, cu_seqlens, dev)
    gp, gs = _mat(_packed(gate, gate, "gate"), dtype, dev, "gate")
    vp, vs = _mat(_packed(value, gate, "value"), dtype, dev, "value")
    dp, ds = _mat(_packed(dy, gate, "dy"), dtype, dev, "dy")
    f32 = torch.float32
    _shaped(states, ((T + STATE_ROWS - 1) // STATE_ROWS, H), "states")
    for name, t in (("initial_state", initial_state), ("dfinal_state", dfinal_state)):
        if t is not None:
            _shaped(t, (B, H), name)
    dgate, dvalue = (torch.empty(gate.shape, dtype=dtype, device=dev) for _ in range(2))
    dinit = None if initial_state is None else torch.empty(B, H, dtype=f32, device=dev)
    ref, nbytes = _desc(dev, ScanDesc, (T, H, B, gs, vs, ds, _dtype_code(dtype, "gate"), _form(kind), 0),
                        "molt_gated_scan_workspace_bytes")
    ws = workspace if workspace is not None else _scratch(nbytes, dev, "gated_scan", stream)
    _call(load().molt_gated_scan_bwd, dev, ref, dp, gp, vp, _vec(states, f32, dev, "states"),
          _vec(initial_state, f32, dev, "initial_state"), cu, _vec(dfinal_state, f32, dev, "dfinal_state"),
          dgate.data_ptr(), dvalue.data_ptr(), dinit if dinit is None else dinit.data_ptr(), ws.data_ptr(), ws.numel(),
          _handle(stream, dev))
    return {"dgate": dgate, "dvalue": dvalue, "dinitial_state": dinit}


@_on_stream
def gated_scan_step(gate, value, state, kind="sigmoid", out_state=None, stream=None):
    """One row of each of B sequences (molt_gated_scan_step), as decoding takes them: gate,
    value [B, H], state [B, H] float32.  Returns dict(y, state): the new state, in `out_state`
    where one is given (it may be `state` itself)."""
    torch = _torch()
    B, H = gate.shape
    dev, dtype = _cuda(gate, "gate"), gate.dtype
    gp, gs = _mat(gate, dtype, dev, "gate")
    vp, vs = _mat(_shaped(value, (B, H), "value"), dtype, dev, "value")
    f32 = torch.float32
    y = torch.empty(B, H, dtype=dtype, device=dev)
    new = torch.empty(B, H, dtype=f32, device=dev) if out_state is None else _shaped(out_state, (B, H), "out_state")
    ref, _ = _desc(dev, ScanDesc, (B, H, B, gs, vs, 0, _dtype_code(dtype, "gate"), _form(kind), 0))
    _call(load().molt_gated_scan_step, dev, ref, gp, vp, _vec(_shaped(state, (B, H), "state"), f32, dev, "state"), y.data_ptr(),
          _vec(new, f32, dev, "out_state"), _handle(stream, dev))
    return {"y": y, "state": new}


# --------------------------------------------------------------------- dropout
def _dropout(x, p, seed, offset, residual, res_scale, first_row, out, out_dtype, stream):
    torch = _torch()
    T, H = x.shape
    dev, dtype = _cuda(x, "x"), x.dtype
    words = None
    if isinstance(seed, torch.Tensor):
        if offset != 0:
            raise ValueError("a seed on the device brings its offset with it")
        words, seed = _vec(_shaped(seed, (2,), "seed"), torch.int64, dev, "seed"), 0
    elif not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise ValueError("seed and offset must be in [0, 2^64)")
    xp, xs = _mat(x, dtype, dev, "x")
    rp = rs = None
    if residual is not None:
        rp, rs = _mat(_shaped(residual, (T, H), "residual"), out_dtype, dev, "residual")
    if out is None:
        out = torch.empty(T, H, dtype=out_dtype, device=dev)
    d = DropoutDesc(T, H, xs, rs or 0, first_row, seed, offset, p, res_scale, _dtype_code(dtype, "x"),
                    _dtype_code(out_dtype, "out"))
    _call(load().molt_dropout, dev, ctypes.byref(d), xp, rp, words, _vec(_shaped(out, (T, H), "out"), out_dtype, dev, "out"),
          _handle(stream, dev))
    return out


@_on_stream
def dropout_fwd(x, p, seed, offset=0, residual=None, res_scale=1.0, first_row=0, out=None, stream=None):
    """res_scale * residual + x with a share p of its elements left out and the others divided
    by 1 - p (molt_dropout); p counts in steps of 2^-16.  The mask is a function of (seed, offset,
    first_row + row, column) and is not stored: the backward gives the same four.  seed: an
    integer, or an int64 CUDA tensor [2] of seed and offset that is read when the kernel runs
    (in a captured graph a program sets it before every replay).  x [T, H], residual [T, H] or
    None of x's type or float32 (x may be float32 beside any); the result has residual's type, or
    x's.  `out` may be x or residual."""
    return _dropout(x, p, seed, offset, residual, res_scale, first_row, out,
                    x.dtype if residual is None else residual.dtype, stream)


@_on_stream
def dropout_bwd(dout, p, seed, offset=0, first_row=0, dtype=None, out=None, stream=None):
    """Gradient of dropout_fwd for x, of dout's type or `dtype` (molt_dropout); the residual's
    is res_scale * dout."""
    return _dropout(dout, p, seed, offset, None, 1.0, first_row, out, dout.dtype if dtype is None else dtype, stream)
