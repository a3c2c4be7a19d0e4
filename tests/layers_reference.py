"""Definitions in 64 bits of the order model's norm, its rows and products in 8 bits and its shaped logits (include/cc.h), for the
tests: plain loops over rows where a definition has them, tensors on any device."""
import math

import torch

U24 = 2.0 ** -24                                       # half a step of fp32
HALF_STEP = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}    # of the last rounding; that of fp32 is counted in U24
BELOW = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}   # half a step of the smallest values


def rounded(want, dtype, error=0.0):
    """How far a result may be from `want` when it is computed to within `error` and rounded to dtype: the rounding is
    of the computed value, so its step is that of |want| + error."""
    return error + HALF_STEP[dtype] * (want.abs() + error) + BELOW[dtype]


def added(x, residual):
    """h: the sum as an element of the type.  A sum of two elements in 64 bits is exact, or so near to it that it rounds alike in 32."""
    return x if residual is None else (x.float() + residual.float()).to(x.dtype)


def norm(h, weight, eps):
    """(out, r) in 64 bits."""
    h64 = h.double()
    r = 1 / torch.sqrt((h64 * h64).mean(-1, keepdim=True) + eps)
    w = torch.ones(h.shape[-1], dtype=torch.float64, device=h.device) if weight is None else weight.double()
    return h64 * r * w, r.squeeze(-1)


def eight_bits(u, r):
    """(q, scale) of rows u in 64 bits that were not multiplied by r."""
    most = u.abs().amax(-1)
    bad = ~torch.isfinite(u).all(-1)
    safe = torch.where((most == 0) | bad, 1.0, most)
    q = torch.round(127 * u / safe.unsqueeze(-1))
    q = torch.where((bad | (most == 0)).unsqueeze(-1), 0.0, q)
    return q, torch.where(bad, math.nan, most * r / 127)


def norm_backward(grad_out, h, weight, r, grad_sum):
    """(grad_h, grad_weight) in 64 bits, from r as the forward call gave it."""
    g, h64, s = grad_out.double(), h.double(), r.double().unsqueeze(-1)
    w = torch.ones(h.shape[-1], dtype=torch.float64, device=h.device) if weight is None else weight.double()
    normed = h64 * s
    grad = s * (g * w - normed * (g * w * normed).mean(-1, keepdim=True))
    if grad_sum is not None:
        grad = grad + grad_sum.double()
    return grad, (g * normed).flatten(0, -2).sum(0)


def product(x, x_scale, w, w_scale, bias):
    """The result in 64 bits; the sum of whole numbers is exact in them."""
    out = (x.double() @ w.double().t().contiguous()) * x_scale.double().unsqueeze(-1) * w_scale.double()
    return out if bias is None else out + bias.double()


def looked_back_on(history, lengths, starts, b, t):
    """The tokens that row (b, t) sees and those of them that count, as lists."""
    if history is None:
        return [], []
    n = min(max((0 if lengths is None else int(lengths[b])) + t, 0), history.shape[1])
    start = 0 if starts is None else int(starts[b])
    row = history[b, :n].tolist()
    return row, [token for i, token in enumerate(row) if i >= start]


def shaped(logits, history=None, lengths=None, penalties=None, starts=None, bias=None, allowed=None):
    """(out, slope, size) in 64 bits on the CPU: the shaped logits, the gradient's factor, and the sum of the sizes of what was
    added up to them."""
    z = logits.cpu().double()
    nb, nt, v = z.shape
    history, lengths, starts, penalties, bias, allowed = (None if a is None else a.cpu() for a in (history, lengths, starts, penalties, bias, allowed))
    out, slope, size = z.clone(), torch.ones_like(z), z.abs()
    for b in range(nb):
        r, p, f = (1.0, 0.0, 0.0) if penalties is None else penalties[b].double().tolist()
        for t in range(nt):
            gone = torch.zeros(v, dtype=torch.bool)
            if penalties is not None:
                seen, counted = looked_back_on(history, lengths, starts, b, t)
                for token in set(seen):
                    if not 0 <= token < v:
                        continue
                    factor = 1 / r if z[b, t, token] > 0 else r
                    slope[b, t, token] = factor
                    out[b, t, token] *= factor
                    size[b, t, token] *= factor
                    count = counted.count(token)
                    if count:
                        out[b, t, token] -= p + f * count
                        size[b, t, token] += abs(p) + abs(f) * count
                        if math.inf in (p, f):
                            gone[token] = True
            if bias is not None:
                row = (bias if bias.dim() == 1 else bias[b]).double()
                out[b, t] += row
                size[b, t] += row.abs()
                gone |= row == -math.inf
            if allowed is not None:
                words = allowed[b, t].long()
                j = torch.arange(v)
                gone |= (words[j // 32] >> (j % 32)) & 1 == 0
            out[b, t, gone] = -math.inf
            slope[b, t, gone] = 0.0
    return out, slope, size
