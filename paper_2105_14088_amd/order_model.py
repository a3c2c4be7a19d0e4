"""Binding of the order model's calls (include/cc.h, from cc_embed on): embedding lookup and gradient, gated recurrence and
gradient, log-probabilities, policy loss, preference loss, norm of a sum and gradient, rows and products in 8 bits, shaped logits and
gradient.

As in binding.py, only arguments are marshalled here: device tensors in, device tensors out, on the current stream or the
one given.  Tensors may be strided as long as their last dimension is contiguous; a tensor made here is contiguous."""
from __future__ import annotations

import functools
from typing import NamedTuple, Optional

import torch

from . import binding as _binding
from .binding import _check, _dev, _new, _stream, lib

CC_MEAN_TOKENS, CC_MEAN_ORDERS = 0, 1
MEANS = {"tokens": CC_MEAN_TOKENS, "orders": CC_MEAN_ORDERS}
CC_SCAN_CHUNK = 16

_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def _dtype(t: torch.Tensor, name: str) -> int:
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, float16 or bfloat16")
    return code


# A small call is bound by what Python does for it: a tensor that is as it should be is looked at once, and what is wrong
# with another is found out afterwards.
def _strided(t: torch.Tensor, shape, dtype, name: str):
    """Where a tensor with a contiguous last dimension lies, and its other strides."""
    strides = t.stride()
    if t.dtype is dtype and t.shape == shape and t.is_cuda and (strides[-1] == 1 or shape[-1] <= 1):
        return (t.data_ptr(), *strides[:-1])
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name} must be {dtype} {list(shape)}")
    raise ValueError(f"{name}'s last dimension must be contiguous")


def _plain(t: Optional[torch.Tensor], shape, dtype, name: str) -> Optional[int]:
    """Where a contiguous tensor lies, or None for none."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}")
    return _dev(t, dtype, name)


# What is made here is not looked at like what is passed in.
def _rows_out(t: Optional[torch.Tensor], shape, dtype, device, stream, name: str):
    """A result [A, B, C] of the caller's or made here, and where it lies with its strides."""
    if t is None:
        t = _new(shape, dtype, device, stream)
        return t, (t.data_ptr(), shape[1] * shape[2], shape[2])
    return t, _strided(t, shape, dtype, name)


def _plain_out(t: Optional[torch.Tensor], shape, dtype, device, stream, name: str):
    """A contiguous result of the caller's or made here, and where it lies."""
    if t is None:
        t = _new(shape, dtype, device, stream)
        return t, t.data_ptr()
    return t, _plain(t, shape, dtype, name)


@functools.lru_cache(maxsize=4096)
def _scan_bytes(b: int, t: int, d: int) -> int:
    return lib().cc_gated_scan_workspace_bytes(b, t, d)


@functools.lru_cache(maxsize=4096)
def _embed_bytes(v: int, d: int, n: int) -> int:
    return lib().cc_embed_workspace_bytes(v, d, n)


@functools.lru_cache(maxsize=4096)
def _token_bytes(b: int, t: int) -> int:
    return lib().cc_token_workspace_bytes(b, t)


def _workspace(workspace: Optional[torch.Tensor], nbytes: int, device, stream):
    """The caller's workspace or one made here; the tensor is returned so that it lives until the call is enqueued."""
    if workspace is None:
        if nbytes == 0:
            return None, None, 0
        workspace = torch.empty_strided((nbytes,), (1,), dtype=torch.uint8, device=device)     # as _new, and 0.5 us shorter
        if stream is not None:
            workspace.record_stream(stream)
        return workspace, workspace.data_ptr(), nbytes
    return workspace, _dev(workspace, torch.uint8, "workspace"), workspace.numel()


# ------------------------------------------------------------------------------------------------------- embedding


def cc_embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, out: Optional[torch.Tensor] = None,
             stream=None) -> torch.Tensor:
    """scale * table[ids], [*ids.shape, D]; ids outside [0, V) give zeros.  An `out` of the caller's is [*ids.shape, D]
    contiguous, or [ids.numel(), D] with rows apart."""
    if table.dim() != 2:
        raise ValueError("table must be [V, D]")
    (v, d), code = table.shape, _dtype(table, "table")
    where, apart = _strided(table, (v, d), table.dtype, "table")
    n = ids.numel()
    if out is None:
        out = _new((*ids.shape, d), table.dtype, table.device, stream)
        to, out_apart = out.data_ptr(), d
    else:
        to, out_apart = _token_rows(out, ids, d, table.dtype, "out")
    _check(lib().cc_embed(where, code, v, d, apart, _dev(ids, torch.int32, "ids"), n, scale, to, out_apart, _stream(stream)),
           "cc_embed")
    return out


def _token_rows(t: torch.Tensor, ids: torch.Tensor, d: int, dtype, name: str):
    if tuple(t.shape) == (*ids.shape, d) and t.is_contiguous():
        return _dev(t, dtype, name), d
    return _strided(t, (ids.numel(), d), dtype, name)


def cc_embed_workspace_bytes(v: int, d: int, n: int) -> int:
    return int(lib().cc_embed_workspace_bytes(v, d, n))


def cc_embed_backward(grad: torch.Tensor, ids: torch.Tensor, vocab: int, scale: float = 1.0,
                      grad_table: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None,
                      workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of cc_embed's table, [vocab, D]: of grad's type if made here, float32 or grad's type if the caller's.
    With accumulate it is added to the caller's."""
    code, d, n = _dtype(grad, "grad"), int(grad.shape[-1]), ids.numel()
    where, apart = _token_rows(grad, ids, d, grad.dtype, "grad")
    if grad_table is None:
        if accumulate:
            raise ValueError("accumulate needs a grad_table to add to")
        grad_table = _new((vocab, d), grad.dtype, grad.device, stream)
        to, to_code, to_apart = grad_table.data_ptr(), code, d
    else:
        to_code = _dtype(grad_table, "grad_table")
        to, to_apart = _strided(grad_table, (vocab, d), grad_table.dtype, "grad_table")
    L = lib()
    held, ws, nbytes = _workspace(workspace, _embed_bytes(vocab, d, n), grad.device, stream)
    _check(L.cc_embed_backward(where, code, n, d, apart, _dev(ids, torch.int32, "ids"), vocab, scale, to, to_code, to_apart,
                               1 if accumulate else 0, ws, nbytes, _stream(stream)), "cc_embed_backward")
    return grad_table


# ------------------------------------------------------------------------------------------------------ recurrence


def cc_gated_scan_workspace_bytes(b: int, t: int, d: int) -> int:
    return int(lib().cc_gated_scan_workspace_bytes(b, t, d))


def cc_gated_scan(x: torch.Tensor, gate: torch.Tensor, h0: Optional[torch.Tensor] = None,
                  lengths: Optional[torch.Tensor] = None, save_states: bool = False, out: Optional[torch.Tensor] = None,
                  last: Optional[torch.Tensor] = None, states: Optional[torch.Tensor] = None, stream=None,
                  workspace: Optional[torch.Tensor] = None):
    """(h, last, states) of x, gate [B, T, D]: h of x's type, last float32 [B, D], states (None without save_states) what
    cc_gated_scan_backward needs.  `last` may be h0 itself: one step of sampling with the state updated in place."""
    if x.dim() != 3:
        raise ValueError("x must be [B, T, D]")
    shape, code = x.shape, _dtype(x, "x")
    b, t, d = shape
    device = x.device
    out, to = _rows_out(out, shape, x.dtype, device, stream, "out")
    last, last_to = _plain_out(last, (b, d), torch.float32, device, stream, "last")
    states_to = None
    if states is not None or save_states:
        states, states_to = _plain_out(states, (b, (t + CC_SCAN_CHUNK - 1) // CC_SCAN_CHUNK, d), torch.float32, device, stream, "states")
    L = lib()
    held, ws, nbytes = _workspace(workspace, _scan_bytes(b, t, d), x.device, stream)
    _check(L.cc_gated_scan(*_strided(x, shape, x.dtype, "x"), *_strided(gate, shape, x.dtype, "gate"), code, b, t, d,
                           _plain(lengths, (b,), torch.int32, "lengths"), _plain(h0, (b, d), torch.float32, "h0"), *to, last_to, states_to, ws, nbytes, _stream(stream)),
           "cc_gated_scan")
    return out, last, states


def cc_gated_scan_backward(x: torch.Tensor, gate: torch.Tensor, states: torch.Tensor, grad_h: torch.Tensor,
                           grad_last: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                           grad_x: Optional[torch.Tensor] = None, grad_gate: Optional[torch.Tensor] = None,
                           grad_h0: Optional[torch.Tensor] = None, stream=None, workspace: Optional[torch.Tensor] = None):
    """(grad_x, grad_gate, grad_h0) from the gradients of h and of the last state; x, gate, lengths and states are
    cc_gated_scan's."""
    if x.dim() != 3:
        raise ValueError("x must be [B, T, D]")
    shape, code = x.shape, _dtype(x, "x")
    b, t, d = shape
    device = x.device
    grad_x, x_to = _rows_out(grad_x, shape, x.dtype, device, stream, "grad_x")
    grad_gate, gate_to = _rows_out(grad_gate, shape, x.dtype, device, stream, "grad_gate")
    grad_h0, h0_to = _plain_out(grad_h0, (b, d), torch.float32, device, stream, "grad_h0")
    kept = (b, (t + CC_SCAN_CHUNK - 1) // CC_SCAN_CHUNK, d)
    L = lib()
    held, ws, nbytes = _workspace(workspace, _scan_bytes(b, t, d), x.device, stream)
    _check(L.cc_gated_scan_backward(*_strided(x, shape, x.dtype, "x"), *_strided(gate, shape, x.dtype, "gate"), code, b, t, d,
                                    _plain(lengths, (b,), torch.int32, "lengths"), _plain(states, kept, torch.float32, "states"),
                                    *_strided(grad_h, shape, x.dtype, "grad_h"), _plain(grad_last, (b, d), torch.float32, "grad_last"),
                                    *x_to, *gate_to, h0_to,
                                    ws, nbytes, _stream(stream)), "cc_gated_scan_backward")
    return grad_x, grad_gate, grad_h0


# ------------------------------------------------------------------------------------------ log-probabilities, losses


class PolicyLoss(NamedTuple):
    """stats float32 [3]: loss, mean divergence, clipped share; logprob float32 [B, T]; grad_logits [B, T, V] or None."""
    stats: torch.Tensor
    logprob: torch.Tensor
    grad_logits: Optional[torch.Tensor]


class PreferenceLoss(NamedTuple):
    """loss float32 []; margin float32 [B / 2]; logprob float32 [B, T]; grad_logits [B, T, V] or None."""
    loss: torch.Tensor
    margin: torch.Tensor
    logprob: torch.Tensor
    grad_logits: Optional[torch.Tensor]


def _logits(logits: torch.Tensor, tokens: torch.Tensor, mask: Optional[torch.Tensor], placed: bool, scale: float):
    """The first arguments of the calls on logits, and [B, T]."""
    if logits.dim() != 3:
        raise ValueError("logits must be [B, T, V]")
    shape, code = logits.shape, _dtype(logits, "logits")
    where, sb, st = _strided(logits, shape, logits.dtype, "logits")
    positions = shape[:2]
    at = None
    if mask is not None:
        if mask.dtype not in (torch.bool, torch.uint8) or mask.shape != positions:
            raise ValueError("mask must be bool or uint8 [B, T]")
        at = _dev(mask, mask.dtype, "mask")
    return (where, code, *shape, sb, st, _plain(tokens, positions, torch.int32, "tokens"), at, 1 if placed else 0, scale), positions


def _gradient(logits: torch.Tensor, grad_logits: Optional[torch.Tensor], stream):
    return _rows_out(grad_logits, logits.shape, logits.dtype, logits.device, stream, "grad_logits")


def cc_token_logprob(logits: torch.Tensor, tokens: torch.Tensor, mask: Optional[torch.Tensor] = None, placed: bool = False,
                     scale: float = 1.0, logprob: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
                     stream=None):
    """(logprob float32 [B, T], rows float32 [B, T, 2]); rows is what cc_token_logprob_backward needs."""
    args, positions = _logits(logits, tokens, mask, placed, scale)
    logprob, logprob_to = _plain_out(logprob, positions, torch.float32, logits.device, stream, "logprob")
    rows, rows_to = _plain_out(rows, (*positions, 2), torch.float32, logits.device, stream, "rows")
    _check(lib().cc_token_logprob(*args, logprob_to, rows_to, _stream(stream)), "cc_token_logprob")
    return logprob, rows


def cc_token_logprob_backward(logits: torch.Tensor, tokens: torch.Tensor, mask: Optional[torch.Tensor], placed: bool,
                              scale: float, rows: torch.Tensor, grad_logprob: torch.Tensor, grad_scale: float = 1.0,
                              grad_logits: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """grad_logits [B, T, V]; the first five arguments are cc_token_logprob's.  `grad_logits` may be the logits."""
    args, positions = _logits(logits, tokens, mask, placed, scale)
    grad_logits, to = _gradient(logits, grad_logits, stream)
    _check(lib().cc_token_logprob_backward(*args, _plain(rows, (*positions, 2), torch.float32, "rows"),
                                           _plain(grad_logprob, positions, torch.float32, "grad_logprob"), grad_scale, *to, _stream(stream)),
           "cc_token_logprob_backward")
    return grad_logits


def cc_token_workspace_bytes(b: int, t: int) -> int:
    return int(lib().cc_token_workspace_bytes(b, t))


def cc_policy_loss(logits: torch.Tensor, tokens: torch.Tensor, old_logprob: torch.Tensor, advantage: torch.Tensor,
                   ref_logprob: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, placed: bool = False,
                   scale: float = 1.0, clip_low: float = 0.2, clip_high: float = 0.2, kl_coef: float = 0.0,
                   mean: str = "tokens", grad_scale: float = 1.0, grad: bool = True,
                   grad_logits: Optional[torch.Tensor] = None, stream=None,
                   workspace: Optional[torch.Tensor] = None) -> PolicyLoss:
    """The clipped policy loss and, unless grad is false, its gradient.  advantage: float32 [B] or [B, T].  mean: "tokens"
    or "orders".  `grad_logits` may be the logits."""
    args, positions = _logits(logits, tokens, mask, placed, scale)
    if mean not in MEANS:
        raise ValueError("mean must be 'tokens' or 'orders'")
    per_token = advantage.dim() == 2
    to = (None, 0, 0)
    if grad:
        grad_logits, to = _gradient(logits, grad_logits, stream)
    stats = _new(3, torch.float32, logits.device, stream)
    logprob = _new(positions, torch.float32, logits.device, stream)
    L = lib()
    held, ws, nbytes = _workspace(workspace, _token_bytes(*positions), logits.device, stream)
    _check(L.cc_policy_loss(*args, _plain(old_logprob, positions, torch.float32, "old_logprob"), _plain(ref_logprob, positions, torch.float32, "ref_logprob"),
                            _plain(advantage, positions if per_token else positions[:1], torch.float32, "advantage"), 1 if per_token else 0,
                            clip_low, clip_high, kl_coef, MEANS[mean], grad_scale, stats.data_ptr(), logprob.data_ptr(), *to,
                            ws, nbytes, _stream(stream)), "cc_policy_loss")
    return PolicyLoss(stats, logprob, grad_logits if grad else None)


def cc_preference_loss(logits: torch.Tensor, tokens: torch.Tensor, ref_logprob: Optional[torch.Tensor] = None,
                       mask: Optional[torch.Tensor] = None, placed: bool = False, scale: float = 1.0, beta: float = 0.1,
                       label_smoothing: float = 0.0, grad_scale: float = 1.0, grad: bool = True,
                       grad_logits: Optional[torch.Tensor] = None, stream=None,
                       workspace: Optional[torch.Tensor] = None) -> PreferenceLoss:
    """The preference loss of the pairs (i, B/2 + i), the first of which is preferred, and, unless grad is false, its
    gradient.  `grad_logits` may be the logits."""
    args, positions = _logits(logits, tokens, mask, placed, scale)
    to = (None, 0, 0)
    if grad:
        grad_logits, to = _gradient(logits, grad_logits, stream)
    loss = _new((), torch.float32, logits.device, stream)
    margin = _new(positions[0] // 2, torch.float32, logits.device, stream)
    logprob = _new(positions, torch.float32, logits.device, stream)
    L = lib()
    held, ws, nbytes = _workspace(workspace, _token_bytes(*positions), logits.device, stream)
    _check(L.cc_preference_loss(*args, _plain(ref_logprob, positions, torch.float32, "ref_logprob"), beta, label_smoothing, grad_scale,
                                loss.data_ptr(), margin.data_ptr(), logprob.data_ptr(), *to, ws, nbytes, _stream(stream)),
           "cc_preference_loss")
    return PreferenceLoss(loss, margin, logprob, grad_logits if grad else None)


# ------------------------------------------------------------------------------------------ norm, rows and products in 8 bits


class RmsNorm(NamedTuple):
    """out: the normalised rows, or None; sum: x + residual (x itself without one); q int8 and scale float32, or None; rstd
    float32, or None.  All of x's shape, scale and rstd without its last dimension."""
    out: Optional[torch.Tensor]
    sum: torch.Tensor
    q: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]
    rstd: Optional[torch.Tensor]


def _rows(t: torch.Tensor, shape, dtype, name: str):
    """Where the rows of a tensor [..., D] lie, and how far apart: contiguous, or [n, D] with rows apart."""
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr(), shape[-1]
    if t.is_cuda and t.dtype is dtype and t.shape == shape and len(shape) != 2:
        raise ValueError(f"{name} must be contiguous, or [n, D] with rows apart")
    return _strided(t, shape, dtype, name)


# torch makes a contiguous tensor like another, or one whose strides are given, in 1.2 us, one of a shape in 2.1: a small call with
# three results takes a fifth less of it.
def _like(t: torch.Tensor, dtype, stream) -> torch.Tensor:
    """A contiguous tensor of t's shape that a call makes, as _new does."""
    if not t.is_contiguous():
        return _new(t.shape, dtype, t.device, stream)
    t = torch.empty_like(t, dtype=dtype)
    if stream is not None:
        t.record_stream(stream)
    return t


def _matrix_new(n: int, d: int, dtype, device, stream) -> torch.Tensor:
    t = torch.empty_strided((n, d), (d, 1), dtype=dtype, device=device)
    if stream is not None:
        t.record_stream(stream)
    return t


def _rows_like(t: Optional[torch.Tensor], x: torch.Tensor, dtype, stream, name: str):
    """Rows of x's shape, the caller's or made here, where they lie and how far apart."""
    if t is None:
        t = _like(x, dtype, stream)
        return t, (t.data_ptr(), x.shape[-1])
    return t, _rows(t, x.shape, dtype, name)


def _each_row(t: Optional[torch.Tensor], x: torch.Tensor, stream, name: str):
    """A number for each of x's rows, the caller's or made here, and where they lie."""
    if t is None:
        lead = x.shape[:-1]
        if len(lead) == 1:
            t = torch.empty_strided((lead[0],), (1,), dtype=torch.float32, device=x.device)
            if stream is not None:
                t.record_stream(stream)
        else:
            t = _new(lead, torch.float32, x.device, stream)
        return t, t.data_ptr()
    return t, _plain(t, x.shape[:-1], torch.float32, name)


@functools.lru_cache(maxsize=None)
def _several_devices() -> bool:
    """Whether a tensor on the GPU can be on another than the current one: looking at all that a small call takes is 3 % of it."""
    return torch.cuda.device_count() > 1


def _stream_at(t: torch.Tensor, stream, *passed: Optional[torch.Tensor]) -> int:
    """The stream's handle.  A kernel is launched on the current device: of t and what else was passed in, on a tensor of another it would read
    what may not be there."""
    current = torch.cuda.current_device() if _binding._current_device is None else _binding._current_device()
    if t.get_device() != current:
        raise ValueError("tensors must be on the current device")
    if _several_devices():
        for other in passed:
            if other is not None and other.get_device() != current:
                raise ValueError("tensors must be on the current device")
        if stream is not None and stream.device_index != current:
            raise ValueError("the stream must be one of the current device")
    if stream is None and _binding._current_raw_stream is not None:
        return _binding._current_raw_stream(current)
    return _stream(stream)


_NOWHERE = (None, 0)


@functools.lru_cache(maxsize=4096)
def _norm_bytes(n: int, d: int) -> int:
    return lib().cc_rms_norm_workspace_bytes(n, d)


@functools.lru_cache(maxsize=4096)
def _product_bytes(m: int, n: int, k: int) -> int:
    return lib().cc_product_i8_workspace_bytes(m, n, k)


def cc_rms_norm_workspace_bytes(n: int, d: int) -> int:
    return int(lib().cc_rms_norm_workspace_bytes(n, d))


def cc_product_i8_workspace_bytes(m: int, n: int, k: int) -> int:
    return int(lib().cc_product_i8_workspace_bytes(m, n, k))


def _weight(weight: Optional[torch.Tensor], d: int, dtype, name: str):
    """Where a weight lies and its type's code."""
    if weight is None:
        return None, _DTYPES[dtype]
    if weight.dtype is not torch.float32 and weight.dtype is not dtype:
        raise ValueError(f"{name} must be float32 or {dtype}")
    return _plain(weight, (d,), weight.dtype, name), _DTYPES[weight.dtype]


def cc_rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, eps: float = 1e-6,
                normed: bool = True, quantized: bool = False, save_rstd: bool = False, out: Optional[torch.Tensor] = None,
                sum: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                rstd: Optional[torch.Tensor] = None, stream=None) -> RmsNorm:
    """The norm of x + residual, [..., D]; `sum` may be x or residual itself.  normed: the rows in x's type; quantized: as int8
    with a scale each, for cc_product_i8; save_rstd: with what cc_rms_norm_backward needs."""
    shape, dtype = x.shape, x.dtype
    code = _dtype(x, "x")
    if not shape:
        raise ValueError("x must be [..., D]")
    passed = (weight, residual, out, sum, q, scale, rstd)
    d = shape[-1]
    n = x.numel() // d if d else 0
    x_at = _rows(x, shape, dtype, "x")
    residual_at = sum_to = out_to = q_to = _NOWHERE
    if residual is not None:
        residual_at = _rows(residual, shape, dtype, "residual")
    if residual is not None or sum is not None:
        sum, sum_to = _rows_like(sum, x, dtype, stream, "sum")
    if normed or out is not None:
        out, out_to = _rows_like(out, x, dtype, stream, "out")
    scale_to = rstd_to = None
    if quantized or q is not None:
        q, q_to = _rows_like(q, x, torch.int8, stream, "q")
        scale, scale_to = _each_row(scale, x, stream, "scale")
    elif scale is not None:
        raise ValueError("scale goes with quantized rows")
    if save_rstd or rstd is not None:
        rstd, rstd_to = _each_row(rstd, x, stream, "rstd")
    _check(lib().cc_rms_norm(*x_at, *residual_at, code, n, d, *_weight(weight, d, dtype, "weight"), eps, *sum_to, *out_to, *q_to,
                             scale_to, rstd_to, _stream_at(x, stream, *passed)), "cc_rms_norm")
    return RmsNorm(out, x if sum is None else sum, q, scale, rstd)


def cc_rms_norm_backward(grad_out: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: Optional[torch.Tensor] = None,
                         grad_sum: Optional[torch.Tensor] = None, grad_h: Optional[torch.Tensor] = None,
                         grad_weight: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None,
                         workspace: Optional[torch.Tensor] = None):
    """(grad_h, grad_weight): h and rstd are cc_rms_norm's sum and rstd, grad_sum the gradient that reaches the sum past the norm.
    grad_h, the gradient of x and of residual alike, may be grad_out or grad_sum itself.  grad_weight (None without a weight) is of
    the weight's type if made here, float32 or the weight's type if the caller's; with accumulate it is added to the caller's."""
    shape, dtype, device = h.shape, h.dtype, h.device
    code = _dtype(h, "h")
    if not shape:
        raise ValueError("h must be [..., D]")
    passed = (grad_out, rstd, weight, grad_sum, grad_h, grad_weight, workspace)
    d = shape[-1]
    n = h.numel() // d if d else 0
    h_at, grad_at = _rows(h, shape, dtype, "h"), _rows(grad_out, shape, dtype, "grad_out")
    sum_at = _NOWHERE if grad_sum is None else _rows(grad_sum, shape, dtype, "grad_sum")
    grad_h, grad_h_to = _rows_like(grad_h, h, dtype, stream, "grad_h")
    to, to_code, held, ws, nbytes = None, code, None, None, 0
    if weight is None:
        if grad_weight is not None:
            raise ValueError("grad_weight goes with a weight")
    else:
        if grad_weight is None:
            if accumulate:
                raise ValueError("accumulate needs a grad_weight to add to")
            grad_weight = _like(weight, weight.dtype, stream)
        to, to_code = _plain(grad_weight, (d,), grad_weight.dtype, "grad_weight"), _dtype(grad_weight, "grad_weight")
        held, ws, nbytes = _workspace(workspace, _norm_bytes(n, d), device, stream)
    _check(lib().cc_rms_norm_backward(*grad_at, *h_at, code, n, d, *_weight(weight, d, dtype, "weight"),
                                      _plain(rstd, shape[:-1], torch.float32, "rstd"), *sum_at, *grad_h_to, to, to_code,
                                      1 if accumulate else 0, ws, nbytes, _stream_at(h, stream, *passed)), "cc_rms_norm_backward")
    return grad_h, grad_weight


def cc_quantize_rows(x: torch.Tensor, q: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None, stream=None):
    """(q int8 [..., D], scale float32 [...]) of x [..., D]: about q * scale."""
    shape, code = x.shape, _dtype(x, "x")
    if not shape:
        raise ValueError("x must be [..., D]")
    passed = (q, scale)
    d = shape[-1]
    x_at = _rows(x, shape, x.dtype, "x")
    q, q_to = _rows_like(q, x, torch.int8, stream, "q")
    scale, scale_to = _each_row(scale, x, stream, "scale")
    _check(lib().cc_quantize_rows(*x_at, code, x.numel() // d if d else 0, d, *q_to, scale_to, _stream_at(x, stream, *passed)),
           "cc_quantize_rows")
    return q, scale


def cc_product_i8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  dtype: torch.dtype = torch.float32, out: Optional[torch.Tensor] = None, stream=None,
                  workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [..., K] times the rows of w [N, K], both int8, with a scale for each row of x and of w: [..., N] of type dtype, or of
    out's if that is given.  bias: float32 [N]."""
    if w.dim() != 2 or not x.shape:
        raise ValueError("x must be [..., K] and w [N, K]")
    shape, (n, k) = x.shape, w.shape
    if shape[-1] != k:
        raise ValueError("x and w must have rows of one length")
    passed = (x_scale, w, w_scale, bias, out, workspace)
    lead = shape[:-1]
    if out is not None:
        dtype = out.dtype
    code = _DTYPES.get(dtype)
    if code is None:
        raise ValueError("dtype must be float32, float16 or bfloat16")
    x_at, w_at = _rows(x, shape, torch.int8, "x"), _rows(w, (n, k), torch.int8, "w")
    m = lead.numel()
    if out is None:
        out = _matrix_new(m, n, dtype, x.device, stream)
        out_to = (out.data_ptr(), n)
        if len(lead) != 1:
            out = out.view(*lead, n)
    else:
        out_to = _rows(out, (*lead, n), dtype, "out")
    L = lib()
    held, ws, nbytes = _workspace(workspace, _product_bytes(m, n, k), x.device, stream)
    _check(L.cc_product_i8(*x_at, _plain(x_scale, lead, torch.float32, "x_scale"), *w_at, _plain(w_scale, (n,), torch.float32, "w_scale"),
                           _plain(bias, (n,), torch.float32, "bias"), m, n, k, *out_to, code, ws, nbytes, _stream_at(x, stream, *passed)),
           "cc_product_i8")
    return out


# -------------------------------------------------------------------------------------------------------- shaped logits


def _shape_args(logits: torch.Tensor, history, lengths, penalties, starts, bias, allowed):
    """The arguments that cc_shape_logits and its gradient share."""
    if logits.dim() != 3:
        raise ValueError("logits must be [B, T, V]")
    shape, code = logits.shape, _dtype(logits, "logits")
    b, t, v = shape
    where, sb, st = _strided(logits, shape, logits.dtype, "logits")
    history_at, length, apart = None, 0, 0
    if history is not None:
        if history.dim() != 2 or history.shape[0] != b:
            raise ValueError("history must be [B, L]")
        if t == 1 and lengths is None:
            raise ValueError("a single position's history needs lengths")
        length = history.shape[1]
        history_at, apart = _strided(history, (b, length), torch.int32, "history")
    bias_at, bias_apart = None, 0
    if bias is not None:
        if bias.shape == (v,):
            bias_at = _plain(bias, (v,), torch.float32, "bias")
        else:
            bias_at, bias_apart = _strided(bias, (b, v), torch.float32, "bias")
    allowed_at = (None, 0, 0)
    if allowed is not None:
        allowed_at = _strided(allowed, (b, t, (v + 31) // 32), torch.int32, "allowed")
    return (where, code, b, t, v, sb, st, history_at, length, apart, _plain(lengths, (b,), torch.int32, "lengths"),
            _plain(starts, (b,), torch.int32, "starts"), _plain(penalties, (b, 3), torch.float32, "penalties"), bias_at, bias_apart,
            *allowed_at)


def _logits_like(t: Optional[torch.Tensor], logits: torch.Tensor, stream, name: str):
    """Logits' shape and type, the caller's or made here, and where they lie with their strides."""
    if t is None:
        t, shape = _like(logits, logits.dtype, stream), logits.shape
        return t, (t.data_ptr(), shape[1] * shape[2], shape[2])
    return t, _strided(t, logits.shape, logits.dtype, name)


def cc_shape_logits(logits: torch.Tensor, history: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
                    penalties: Optional[torch.Tensor] = None, starts: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                    allowed: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Logits [B, T, V] with penalties float32 [B, 3] (repetition, presence, frequency) on the tokens of history int32 [B, L] that a row
    looks back on, bias float32 [V] or [B, V], and allowed int32 [B, T, ceil(V / 32)], a bit for each token.  Row t looks
    back on the first lengths[b] + t entries; without lengths on the first t, as when the history is the orders themselves.
    `out` may be the logits."""
    args = _shape_args(logits, history, lengths, penalties, starts, bias, allowed)
    passed = (history, lengths, penalties, starts, bias, allowed, out)
    out, to = _logits_like(out, logits, stream, "out")
    _check(lib().cc_shape_logits(*args, *to, _stream_at(logits, stream, *passed)), "cc_shape_logits")
    return out


def cc_shape_logits_backward(grad_out: torch.Tensor, logits: torch.Tensor, history: Optional[torch.Tensor] = None,
                             lengths: Optional[torch.Tensor] = None, penalties: Optional[torch.Tensor] = None,
                             starts: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                             allowed: Optional[torch.Tensor] = None, grad_logits: Optional[torch.Tensor] = None,
                             stream=None) -> torch.Tensor:
    """The gradient of the logits from that of cc_shape_logits's result, whose arguments the others are.  `grad_logits` may be
    grad_out."""
    args = _shape_args(logits, history, lengths, penalties, starts, bias, allowed)
    passed = (grad_out, history, lengths, penalties, starts, bias, allowed, grad_logits)
    grad_logits, to = _logits_like(grad_logits, logits, stream, "grad_logits")
    _check(lib().cc_shape_logits_backward(*_strided(grad_out, logits.shape, logits.dtype, "grad_out"), *args, *to,
                                          _stream_at(logits, stream, *passed)), "cc_shape_logits_backward")
    return grad_logits
