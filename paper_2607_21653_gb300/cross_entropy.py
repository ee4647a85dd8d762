"""Softmax cross entropy over the LM head (molt_cross_entropy_*): argument marshalling
into the C ABI, as in the rest of the binding."""
from __future__ import annotations

import ctypes

from . import _bf16_bits, _check, _ptr, _stream, _torch, _workspace, load
from .stream import _dtype_code, _same_device, _shaped


class CrossEntropyOptions(ctypes.Structure):
    """molt_ce_options."""
    _fields_ = [("ignore_index", ctypes.c_int64), ("label_smoothing", ctypes.c_float), ("z_loss", ctypes.c_float)]


def _prepare(hidden, weight, targets, token_weight):
    T, H = hidden.shape
    V, Hw = weight.shape
    if Hw != H:
        raise ValueError(f"weight must have shape [V, {H}], got {list(weight.shape)}")
    _shaped(targets, (T,), "targets")
    if token_weight is not None:
        _shaped(token_weight, (T,), "token_weight")
    _same_device(hidden.device, weight=weight, targets=targets, token_weight=token_weight)
    return T, H, V


def cross_entropy_fwd(hidden, weight, targets, token_weight=None, denom=0.0, ignore_index=-100, label_smoothing=0.0,
                      z_loss=0.0, want_token_outputs=True, stream=None, workspace=None):
    """Cross entropy of the next token over the LM head, without its gradient
    (evaluation).  hidden [T, H], weight [V, H] bf16, targets [T] int32, token_weight [T]
    fp32 or None.  Returns dict(loss [1], logp, lse [T] fp32 (None unless
    want_token_outputs; 0 on ignored rows), stats [5 x 8 bytes])."""
    torch = _torch()
    T, H, V = _prepare(hidden, weight, targets, token_weight)
    dev, f32 = hidden.device, torch.float32
    out = {"loss": torch.empty(1, dtype=f32, device=dev),
           "logp": torch.empty(T, dtype=f32, device=dev) if want_token_outputs else None,
           "lse": torch.empty(T, dtype=f32, device=dev) if want_token_outputs else None,
           "stats": torch.empty(5, dtype=torch.float64, device=dev)}
    opts = CrossEntropyOptions(int(ignore_index), float(label_smoothing), float(z_loss))
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(int(L.molt_cross_entropy_workspace_bytes(T, H, V, 0, 2)), dev, "cross_entropy_fwd", stream)
    _check(L.molt_cross_entropy_fwd(
        _bf16_bits(hidden, "hidden"), _bf16_bits(weight, "weight"), _ptr(targets, torch.int32, "targets"),
        _ptr(token_weight, f32, "token_weight"), T, H, V, float(denom), ctypes.byref(opts), _ptr(out["loss"]),
        _ptr(out["logp"]), _ptr(out["lse"]), _ptr(out["stats"]), ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return out


def cross_entropy_fwd_bwd(hidden, weight, targets, token_weight=None, denom=0.0, ignore_index=-100,
                          label_smoothing=0.0, z_loss=0.0, dW=None, accumulate_dW=False, dW_dtype=None,
                          want_token_outputs=True, stream=None, workspace=None):
    """Cross entropy of the next token over the LM head with its gradient, the [T, V]
    logits never kept.  As cross_entropy_fwd, and dhidden [T, H] bf16 and dW [V, H]: fp32,
    or `dW_dtype` = bfloat16.  With `dW` it is written there, with accumulate_dW (fp32)
    added."""
    torch = _torch()
    T, H, V = _prepare(hidden, weight, targets, token_weight)
    dev, f32 = hidden.device, torch.float32
    if dW is None:
        dW = torch.empty(V, H, dtype=f32 if dW_dtype is None else dW_dtype, device=dev)
        accumulate_dW = False
    else:
        _shaped(dW, (V, H), "dW")
        _same_device(dev, dW=dW)
    out = {"loss": torch.empty(1, dtype=f32, device=dev),
           "logp": torch.empty(T, dtype=f32, device=dev) if want_token_outputs else None,
           "lse": torch.empty(T, dtype=f32, device=dev) if want_token_outputs else None,
           "stats": torch.empty(5, dtype=torch.float64, device=dev),
           "dhidden": torch.empty(T, H, dtype=torch.bfloat16, device=dev), "dW": dW}
    code = _dtype_code(dW.dtype, "dW")
    opts = CrossEntropyOptions(int(ignore_index), float(label_smoothing), float(z_loss))
    L = load()
    ws = workspace
    if ws is None:
        ws = _workspace(int(L.molt_cross_entropy_workspace_bytes(T, H, V, 1, code)), dev, "cross_entropy", stream)
    _check(L.molt_cross_entropy_fwd_bwd(
        _bf16_bits(hidden, "hidden"), _bf16_bits(weight, "weight"), _ptr(targets, torch.int32, "targets"),
        _ptr(token_weight, f32, "token_weight"), T, H, V, float(denom), ctypes.byref(opts), _ptr(out["loss"]),
        _ptr(out["dhidden"]), _ptr(dW, dW_dtype, "dW"), code, 1 if accumulate_dW else 0, _ptr(out["logp"]),
        _ptr(out["lse"]), _ptr(out["stats"]), ws.data_ptr(), ws.numel(), _stream(stream, dev.index)))
    return out


def cross_entropy_stats(stats_tensor) -> dict:
    """Decode molt_ce_stats, copied to the host."""
    raw = stats_tensor.detach().cpu()
    torch = _torch()
    d = raw.tolist()
    return {"denom": d[0], "loss": d[1], "sum_nll": d[2], "sum_lse_sq": d[3],
            "n_active": int(raw.view(torch.int64)[4])}
