"""Binding of the order model's calls (include/cc.h, from cc_embed on): embedding lookup and gradient, gated recurrence and
gradient, log-probabilities, policy loss, preference loss.

As in binding.py, only arguments are marshalled here: device tensors in, device tensors out, on the current stream or the
one given.  Tensors may be strided as long as their last dimension is contiguous; a tensor made here is contiguous."""
from __future__ import annotations

import functools
from typing import NamedTuple, Optional

import torch

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
        workspace = _new(nbytes, torch.uint8, device, stream)
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
