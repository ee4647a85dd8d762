"""Softmax cross entropy over the LM head (molt_cross_entropy_*): argument marshalling
into the C ABI, as in the rest of the binding."""
from __future__ import annotations

import ctypes

from . import _check, _on_stream, _stream, _torch, _workspace, load
from .stream import _at, _cuda, _dtype_code, _shaped


class CrossEntropyOptions(ctypes.Structure):
    """molt_ce_options."""
    _fields_ = [("ignore_index", ctypes.c_int64), ("label_smoothing", ctypes.c_float), ("z_loss", ctypes.c_float),
                ("max_kept_bytes", ctypes.c_int64)]


_options_cache: dict = {}


def _options(ignore_index, label_smoothing, z_loss, max_kept_bytes=None):
    """Reference to the molt_ce_options of these values (read only)."""
    key = (ignore_index, label_smoothing, z_loss, max_kept_bytes)
    ref = _options_cache.get(key)
    if ref is None:
        if len(_options_cache) >= 64:
            _options_cache.clear()
        if max_kept_bytes is not None and max_kept_bytes < 0:
            raise ValueError("max_kept_bytes must be None or >= 0")
        kept = 0 if max_kept_bytes is None else min(max_kept_bytes, 1 << 62) or -1   # the C side's 0 is its default
        ref = _options_cache[key] = ctypes.byref(CrossEntropyOptions(ignore_index, label_smoothing, z_loss, kept))
    return ref


def _prepare(hidden, weight, targets, token_weight):
    T, H = hidden.shape
    V, Hw = weight.shape
    if Hw != H:
        raise ValueError(f"weight must have shape [V, {H}], got {list(weight.shape)}")
    _shaped(targets, (T,), "targets")
    if token_weight is not None:
        _shaped(token_weight, (T,), "token_weight")
    return T, H, V


@_on_stream
def cross_entropy_fwd(hidden, weight, targets, token_weight=None, denom=0.0, ignore_index=-100, label_smoothing=0.0,
                      z_loss=0.0, want_token_outputs=True, stream=None, workspace=None):
    """Cross entropy of the next token over the LM head, without its gradient
    (evaluation).  hidden [T, H], weight [V, H] bf16, targets [T] int32, token_weight [T]
    fp32 or None.  Returns dict(loss [1], logp, lse [T] fp32 (None unless
    want_token_outputs; 0 on ignored rows), stats [5 x 8 bytes])."""
    torch = _torch()
    T, H, V = _prepare(hidden, weight, targets, token_weight)
    dev = _cuda(hidden, "hidden")
    f32, bf16 = torch.float32, torch.bfloat16
    loss = torch.empty(1, dtype=f32, device=dev)
    stats = torch.empty(5, dtype=torch.float64, device=dev)
    logp = lse = None
    if want_token_outputs:
        logp, lse = torch.empty(T, dtype=f32, device=dev), torch.empty(T, dtype=f32, device=dev)
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(L.molt_cross_entropy_workspace_bytes(T, H, V, 0, 2), dev, "cross_entropy_fwd", stream)
    _check(L.molt_cross_entropy_fwd(
        _at(hidden, bf16, dev, "hidden"), _at(weight, bf16, dev, "weight"), _at(targets, torch.int32, dev, "targets"),
        _at(token_weight, f32, dev, "token_weight"), T, H, V, denom, _options(ignore_index, label_smoothing, z_loss),
        loss.data_ptr(), _at(logp, f32, dev, "logp"), _at(lse, f32, dev, "lse"), stats.data_ptr(), ws.data_ptr(),
        ws.numel(), _stream(stream, dev.index)))
    return {"loss": loss, "logp": logp, "lse": lse, "stats": stats}


@_on_stream
def cross_entropy_fwd_bwd(hidden, weight, targets, token_weight=None, denom=0.0, ignore_index=-100,
                          label_smoothing=0.0, z_loss=0.0, dW=None, accumulate_dW=False, dW_dtype=None,
                          want_token_outputs=True, stream=None, workspace=None, max_kept_bytes=None):
    """Cross entropy of the next token over the LM head with its gradient, without a [T, V]
    tensor of logits or of their gradient in 32 or 16-bit floats.  From H = 640 on the
    workspace holds logits between forward and backward as 16-bit steps, 2.1 bytes each, up
    to max_kept_bytes (None: 4 GB; T = 8192, V = 151936: 2.6 GB); max_kept_bytes = 0
    keeps none, forms every logit twice and takes a quarter more time or so.  As
    cross_entropy_fwd, and dhidden [T, H] bf16 and dW [V, H]: fp32, or `dW_dtype` =
    bfloat16.  With `dW` it is written there, with accumulate_dW (fp32) added."""
    torch = _torch()
    T, H, V = _prepare(hidden, weight, targets, token_weight)
    if dW is not None:
        _shaped(dW, (V, H), "dW")
    dev = _cuda(hidden, "hidden")
    f32, bf16 = torch.float32, torch.bfloat16
    if dW is None:
        dW = torch.empty(V, H, dtype=f32 if dW_dtype is None else dW_dtype, device=dev)
        accumulate_dW = False
    code = _dtype_code(dW.dtype, "dW")
    opts = _options(ignore_index, label_smoothing, z_loss, max_kept_bytes)
    loss = torch.empty(1, dtype=f32, device=dev)
    stats = torch.empty(5, dtype=torch.float64, device=dev)
    dhidden = torch.empty(T, H, dtype=bf16, device=dev)
    logp = lse = None
    if want_token_outputs:
        logp, lse = torch.empty(T, dtype=f32, device=dev), torch.empty(T, dtype=f32, device=dev)
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(L.molt_cross_entropy_workspace_bytes_ex(T, H, V, 1, code, opts), dev, "cross_entropy", stream)
    _check(L.molt_cross_entropy_fwd_bwd(
        _at(hidden, bf16, dev, "hidden"), _at(weight, bf16, dev, "weight"), _at(targets, torch.int32, dev, "targets"),
        _at(token_weight, f32, dev, "token_weight"), T, H, V, denom, opts,
        loss.data_ptr(), dhidden.data_ptr(), _at(dW, dW_dtype or dW.dtype, dev, "dW"), code, 1 if accumulate_dW else 0,
        _at(logp, f32, dev, "logp"), _at(lse, f32, dev, "lse"), stats.data_ptr(), ws.data_ptr(), ws.numel(),
        _stream(stream, dev.index)))
    return {"loss": loss, "logp": logp, "lse": lse, "stats": stats, "dhidden": dhidden, "dW": dW}


def cross_entropy_stats(stats_tensor) -> dict:
    """Decode molt_ce_stats, copied to the host."""
    raw = stats_tensor.detach().cpu()
    torch = _torch()
    d = raw.tolist()
    return {"denom": d[0], "loss": d[1], "sum_nll": d[2], "sum_lse_sq": d[3],
            "n_active": int(raw.view(torch.int64)[4])}
