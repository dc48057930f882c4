"""Losses over the output layer, with their gradients: ctypes mirror of wind_label_loss, wind_distill_loss and
wind_transducer_loss (include/wind.h says what they compute).  Argument checks and output tensors only.

The output layer is given as tensors on the GPU: w_out [V1, H] in float32 or bfloat16 and b_out [V1] in float32 or None, blank the last
output.  Rows have w_out's type (bfloat16 also rounds the logits' gradient before its products: include/wind.h).  Every tensor of a call lies on one device; the kernels are enqueued on that device's current
stream, and nothing waits, allocates outside torch or comes back to the host, so calls can be captured into graphs.

Each function returns the losses, or, with `grad` (names of the inputs whose gradients are wanted), a tuple of the losses and
those gradients in the order asked for: the gradients of sum(weights * losses), `weights` None counting as ones.

There is no autograd graph behind either: hand the gradients on (`torch.autograd.backward((e, p), (de, dp))`, or to the optimiser).  A call without `grad` on tensors
that require gradients is refused where autograd records, since its losses would silently be constants; score under `torch.no_grad()`.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Sequence

from .binding import WIND_BF16, WIND_F32, OutputLayer, _check, load_library


def _ptr(t):
    return None if t is None else t.data_ptr()


def _take(t, name, shape, dtype, device, dense=True):
    """Checks one argument; None passes."""
    if t is None:
        return
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {str(dtype)[6:]} of shape {tuple(shape)}, got {str(t.dtype)[6:]} of shape {tuple(t.shape)}")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must be on the GPU of the other arguments")
    if dense:
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    elif t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s last axis must be contiguous")


def _layer(w_out, b_out):
    import torch

    if w_out.dim() != 2 or w_out.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError("w_out must be a float32 or bfloat16 matrix")
    V1, H = w_out.shape
    device = w_out.device
    _take(w_out, "w_out", (V1, H), w_out.dtype, device, dense=False)
    _take(b_out, "b_out", (V1,), torch.float32, device)
    stride = w_out.stride(0) if V1 > 1 else H
    if stride < H:
        raise ValueError("w_out's rows must not overlap")
    return OutputLayer(_ptr(w_out), _ptr(b_out), stride, V1, H,
                       WIND_BF16 if w_out.dtype == torch.bfloat16 else WIND_F32)


def _on(device):
    """The device of a call as the current one."""
    import torch

    return torch.cuda.device(device) if device.index != torch.cuda.current_device() else contextlib.nullcontext()


def _asked(grad, names, inputs):
    import torch

    grad = tuple(grad or ())
    if any(g not in names for g in grad) or len(set(grad)) != len(grad):
        raise ValueError(f"grad takes each of {names} at most once")
    if not grad and torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in inputs):
        raise ValueError("the losses have no autograd graph: ask for gradients with grad=..., or call under torch.no_grad()")
    return grad


def _row_loss(kind, h, w_out, b_out, labels, logits, temperature, weights, grad):
    import torch

    grad, layer = _asked(grad, ("h", "w", "b"), (h, w_out, b_out, logits, weights)), _layer(w_out, b_out)
    (V1, H), device = w_out.shape, w_out.device
    if h.dim() != 2 or labels.dim() != (1 if kind == "label" else 2):
        raise ValueError("h must be [N, H], labels [N], teacher labels [N, K]")
    N = h.shape[0]
    _take(h, "h", (N, H), w_out.dtype, device, dense=False)
    K = 1 if kind == "label" else int(labels.shape[1])
    _take(labels, "labels", (N,) if kind == "label" else (N, K), torch.int32, device)
    _take(logits, "teacher_logits", (N, K), torch.float32, device)
    _take(weights, "weights", (N,), torch.float32, device)
    stride = int(h.stride(0)) if N > 1 else H
    if stride < H:
        raise ValueError("h's rows must not overlap")
    lib = load_library()
    with _on(device):
        size = C.c_size_t(0)
        _check(lib.wind_row_loss_workspace_bytes(C.byref(layer), N, K, 1 if grad else 0, C.byref(size)))
        workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
        loss = torch.empty(N, dtype=torch.float32, device=device)
        out = {"h": (N, H), "w": (V1, H), "b": (V1,)}
        out = {g: torch.empty(out[g], dtype=torch.float32 if g == "b" else w_out.dtype, device=device) for g in grad}
        tail = (_ptr(weights), N, _ptr(loss), _ptr(out.get("h")), _ptr(out.get("w")), _ptr(out.get("b")), _ptr(workspace), size.value,
                torch.cuda.current_stream(device).cuda_stream)
        if kind == "label":
            _check(lib.wind_label_loss(C.byref(layer), _ptr(h), stride, _ptr(labels), *tail))
        else:
            _check(lib.wind_distill_loss(C.byref(layer), _ptr(h), stride, _ptr(labels), _ptr(logits), K, float(temperature), *tail))
    return (loss, *(out[g] for g in grad)) if grad else loss


def label_loss(h, w_out, b_out, labels, weights=None, grad: Optional[Sequence[str]] = None):
    """Cross entropy of the rows h [N, H] with their labels [N] (int32; negative: the row is left out).  grad: of "h", "w", "b"."""
    return _row_loss("label", h, w_out, b_out, labels, None, 1.0, weights, grad)


def distill_loss(h, w_out, b_out, teacher_labels, teacher_logits, temperature: float = 1.0, weights=None,
                 grad: Optional[Sequence[str]] = None):
    """Distance of the rows h [N, H] from a teacher's K largest logits (teacher_labels int32, teacher_logits float32, both [N, K]; negative
    labels and logits of -inf: not there).  grad: of "h", "w", "b"."""
    if teacher_logits is None:
        raise ValueError("teacher_logits is missing")
    return _row_loss("distill", h, w_out, b_out, teacher_labels, teacher_logits, temperature, weights, grad)


def transducer_loss(e, p, w_out, b_out, labels, frames, label_counts, weights=None, grad: Optional[Sequence[str]] = None):
    """-log P(labels | frames) per utterance, for encoder halves e [B, T, H] and prediction halves p [B, U + 1, H] of the joiner, labels
    [B, U], frames [B] and label_counts [B] (all int32).  grad: of "e", "p", "w", "b"."""
    import torch

    grad, layer = _asked(grad, ("e", "p", "w", "b"), (e, p, w_out, b_out, weights)), _layer(w_out, b_out)
    (V1, H), device = w_out.shape, w_out.device
    if e.dim() != 3 or p.dim() != 3 or labels.dim() != 2 or p.shape[1] < 1:
        raise ValueError("e must be [B, T, H], p [B, U + 1, H] and labels [B, U]")
    B, T, U = int(e.shape[0]), int(e.shape[1]), int(p.shape[1]) - 1
    _take(e, "e", (B, T, H), w_out.dtype, device, dense=False)
    _take(p, "p", (B, U + 1, H), w_out.dtype, device, dense=False)
    _take(labels, "labels", (B, U), torch.int32, device)
    _take(frames, "frames", (B,), torch.int32, device)
    _take(label_counts, "label_counts", (B,), torch.int32, device)
    _take(weights, "weights", (B,), torch.float32, device)
    lib = load_library()
    with _on(device):
        size = C.c_size_t(0)
        _check(lib.wind_transducer_loss_workspace_bytes(C.byref(layer), B, T, U, 1 if grad else 0, C.byref(size)))
        workspace = torch.empty(size.value, dtype=torch.uint8, device=device)
        loss = torch.empty(B, dtype=torch.float32, device=device)
        out = {"e": (B, T, H), "p": (B, U + 1, H), "w": (V1, H), "b": (V1,)}
        out = {g: torch.empty(out[g], dtype=torch.float32 if g == "b" else w_out.dtype, device=device) for g in grad}
        _check(lib.wind_transducer_loss(C.byref(layer), _ptr(e), int(e.stride(0)), int(e.stride(1)), _ptr(p), int(p.stride(0)), int(p.stride(1)),
                                        _ptr(labels), _ptr(frames), _ptr(label_counts), _ptr(weights), B, T, U, _ptr(loss), _ptr(out.get("e")),
                                        _ptr(out.get("p")), _ptr(out.get("w")), _ptr(out.get("b")), _ptr(workspace), size.value,
                                        torch.cuda.current_stream(device).cuda_stream))
    return (loss, *(out[g] for g in grad)) if grad else loss
