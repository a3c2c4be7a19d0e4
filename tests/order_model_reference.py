"""The order model's operators in 64 bits on the CPU, written from their definitions, and bounds on what a computation in
32 bits may be off them.  A bound counts roundings: u = 2^-24 is half a step of 32-bit floats at 1, a result in fewer bits is
off by half a step of its type more (`finish`)."""
import math

import torch

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def finish(ref, err, dtype):
    """Bound of a result that was computed to within err and then rounded to dtype once."""
    info = torch.finfo(dtype)
    half = info.eps / 2 if dtype is not torch.float32 else 0.0
    return err + (ref.abs() + err) * half + info.smallest_normal * info.eps


def within(got, ref, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    same = (got == ref) | (got.isnan() & ref.isnan())
    bad = ~(((got - ref).abs() <= bound) | same)
    if bad.any():
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; at {i}: {float(got[i])!r} for {float(ref[i])!r}, "
                             f"bound {float(bound[i] if bound.shape == ref.shape else bound):.3g}")


# ------------------------------------------------------------------------------------------------------- embedding


def embed(table, ids, scale):
    out = torch.zeros(*ids.shape, table.shape[1], dtype=torch.float64)
    for at in range(ids.numel()):
        i = int(ids.reshape(-1)[at])
        if 0 <= i < table.shape[0]:
            out.view(-1, table.shape[1])[at] = table[i].double() * scale
    return out


def embed_backward(grad, ids, vocab, scale, old=None):
    """The gradient, and the bound: c additions of c terms, a product, perhaps one addition more."""
    flat, rows = ids.reshape(-1).long(), grad.reshape(ids.numel(), -1).double()
    real = (flat >= 0) & (flat < vocab)
    out = torch.zeros(vocab, rows.shape[1], dtype=torch.float64)
    size, count = torch.zeros_like(out), torch.zeros(vocab, 1, dtype=torch.float64)
    out.index_add_(0, flat[real], rows[real])
    size.index_add_(0, flat[real], rows[real].abs())
    count.index_add_(0, flat[real], torch.ones(int(real.sum()), 1, dtype=torch.float64))
    out, err = out * scale, size * abs(scale) * (count + 2) * U
    if old is not None:
        out = out + old.double()
        err = err + out.abs() * U
    return out, err


# ------------------------------------------------------------------------------------------------------ recurrence


def scan(x, gate, h0, lengths):
    """h, last and their bounds.  A sigmoid in 32 bits: the product with log2 e and its rounding (1.5 |g| u), the
    exponential's and the reciprocal's last bit (2u each), a sum and a product (u each); a step adds a product's and a sum's.
    Twice that, since a segment's product of gates stands for its steps where the positions are split."""
    x, gate = x.double(), gate.double()
    b, t, d = x.shape
    n = torch.full((b, 1), t) if lengths is None else lengths.long().clamp(0, t).unsqueeze(1)
    h = torch.zeros(b, d, dtype=torch.float64) if h0 is None else h0.double().clone()
    err = torch.zeros_like(h)
    out, errs = torch.zeros(b, t, d, dtype=torch.float64), torch.zeros(b, t, d, dtype=torch.float64)
    for i in range(t):
        keep, take, eps = _gates(gate[:, i])
        inside = n > i
        new = keep * h + take * x[:, i]
        grown = keep * err + (keep * h.abs() + take * x[:, i].abs()) * eps
        h, err = torch.where(inside, new, h), torch.where(inside, grown, err)
        out[:, i], errs[:, i] = torch.where(inside, h, 0.0), torch.where(inside, err, 0.0)
    return out, h, errs, err


def _gates(g):
    eps = 2 * (1.5 * g.abs().clamp(max=200) + 10) * U
    return torch.sigmoid(g), torch.sigmoid(-g), eps


def scan_backward(x, gate, h0, lengths, grad_h, grad_last):
    """(grad_x, grad_gate, grad_h0) and their bounds."""
    h, _, h_err, _ = scan(x, gate, h0, lengths)
    x, gate, grad_h = x.double(), gate.double(), grad_h.double()
    b, t, d = x.shape
    n = torch.full((b, 1), t) if lengths is None else lengths.long().clamp(0, t).unsqueeze(1)
    zero = torch.zeros(b, d, dtype=torch.float64)
    start = zero if h0 is None else h0.double()
    f = zero.clone() if grad_last is None else grad_last.double().clone()
    f_err = zero.clone()
    dx, dg = torch.zeros_like(x), torch.zeros_like(x)
    dx_err, dg_err = torch.zeros_like(x), torch.zeros_like(x)
    for i in range(t - 1, -1, -1):
        inside = n > i
        keep, take, eps = _gates(gate[:, i])
        before, before_err = (h[:, i - 1], h_err[:, i - 1]) if i > 0 else (start, zero)
        lam = grad_h[:, i] + f
        lam_err = f_err + (grad_h[:, i].abs() + f.abs()) * U
        gap, gap_err = before - x[:, i], before_err + (before.abs() + x[:, i].abs()) * U
        dx[:, i] = torch.where(inside, take * lam, 0.0)
        dx_err[:, i] = take * (lam_err + lam.abs() * eps)
        dg[:, i] = torch.where(inside, keep * take * lam * gap, 0.0)
        dg_err[:, i] = keep * take * (lam_err * gap.abs() + lam.abs() * gap_err + lam_err * gap_err + 2 * lam.abs() * gap.abs() * eps)
        f, f_err = torch.where(inside, keep * lam, f), torch.where(inside, keep * (lam_err + lam.abs() * eps), f_err)
    return (dx, dg, f), (dx_err, dg_err, f_err)


# ------------------------------------------------------------------------------------------ log-probabilities, losses


def counted(tokens, mask, v):
    ok = (tokens >= 0) & (tokens < v)
    return ok if mask is None else ok & mask.bool()


def rows(logits, tokens, mask, placed, scale):
    """Per position: probabilities of the candidates, one minus the token's, log-probability; and how far, relative to
    themselves, probabilities may be off (log-probabilities: as much absolutely).
    An exponential's argument is one fma of which the result's rounding counts (at most 1.5 |z - m| u with that of the product
    with log2 e), its own last bit 2u; V terms are added by lanes, at least 8 of them and at most 1024, then over lanes; a
    quotient and two products more.  The arguments that matter are those of terms not yet below 2^-24 of the sum."""
    logits = logits.double()
    b, t, v = logits.shape
    valid = counted(tokens, mask, v)
    p = torch.zeros(b, t, v, dtype=torch.float64)
    rest = torch.zeros(b, t, dtype=torch.float64)
    lp = torch.zeros(b, t, dtype=torch.float64)
    for i in range(b):
        gone = torch.zeros(v, dtype=torch.bool)
        for j in range(t):
            k = int(tokens[i, j])
            if bool(valid[i, j]):
                in_play = ~gone if placed else torch.ones(v, dtype=torch.bool)
                in_play[k] = True
                z = torch.where(in_play, logits[i, j] * scale, -math.inf)
                m = z.max()
                if m == -math.inf:
                    lp[i, j] = -math.inf
                else:
                    e = torch.exp(z - m)
                    others = e.sum() - e[k] if e[k] < 0.5 else torch.cat([e[:k], e[k + 1:]]).sum()
                    total = others + e[k]
                    p[i, j], rest[i, j] = e / total, others / total
                    lp[i, j] = -torch.log1p(others / e[k]) if others < e[k] else (z[k] - m) - torch.log(total)
            if placed and 0 <= k < v:
                gone[k] = True
    terms = min(v, max(4, v // 8 if v <= 64 else v // 64 + 64))
    return p, rest, lp, valid, (1.5 * 40 + terms + 20) * U


def grad_logits(p, rest, tokens, valid, pull):
    """pull [B, T]: scale * grad_scale * d loss / d logprob."""
    pull = torch.where(valid, pull, 0.0).unsqueeze(2)
    out = -pull * p
    k = tokens.clamp(0, p.shape[2] - 1).long().unsqueeze(2)
    out = out.scatter(2, k, pull * rest.unsqueeze(2))
    return torch.where(valid.unsqueeze(2), out, 0.0)


def policy(lp, valid, old, ref, advantage, clip_low, clip_high, kl_coef, mean):
    """stats [3], the slope of each log-probability, and both per unit of log-probability error: what lp's error does."""
    n = valid.double().sum(1, keepdim=True)
    if mean == "tokens":
        w = valid.double() / max(1.0, float(n.sum()))
    else:
        w = valid.double() / n.clamp(min=1) / max(1.0, float((n > 0).sum()))
    a = (advantage if advantage.dim() == 2 else advantage.unsqueeze(1).expand_as(lp)).double()
    r = torch.exp(torch.where(valid, lp - old.double(), 0.0))
    free, held = r * a, r.clamp(1 - clip_low, 1 + clip_high) * a
    clipped = held < free
    gain = torch.where(clipped, held, free)
    kl = torch.zeros_like(lp)
    slope = torch.where(clipped, 0.0, -free)
    moved = free.abs()
    if ref is not None:
        away = torch.where(valid, ref.double() - lp, 0.0)
        kl = torch.expm1(away) - away
        slope = slope - kl_coef * torch.expm1(away)
        moved = moved + abs(kl_coef) * torch.exp(away) * (1 + away.abs())
    stats = torch.stack([torch.where(valid, w * (kl_coef * kl - gain), 0.0).sum(), torch.where(valid, w * kl, 0.0).sum(),
                         torch.where(valid, w * clipped, 0.0).sum()])
    return stats, torch.where(valid, w * slope, 0.0), torch.where(valid, w * moved, 0.0), torch.where(valid, w * (moved + kl.abs() * abs(kl_coef)), 0.0).sum()


def preference(lp, valid, ref, beta, smoothing):
    """loss, margins, slopes."""
    pairs = lp.shape[0] // 2
    gap = torch.where(valid, lp - (0 if ref is None else ref.double()), 0.0).sum(1)
    m = beta * (gap[:pairs] - gap[pairs:])
    soft = torch.nn.functional.softplus
    loss = ((1 - smoothing) * soft(-m) + smoothing * soft(m)).sum() / max(1, pairs)
    s = beta / max(1, pairs) * (smoothing * torch.sigmoid(m) - (1 - smoothing) * torch.sigmoid(-m))
    return loss, m, torch.cat([s, -s]).unsqueeze(1).expand_as(lp)


def rows_at_once(logits, tokens, mask, placed, scale):
    """What `rows` gives, for all positions together: for many of them."""
    z = logits.double() * scale
    b, t, v = z.shape
    valid = counted(tokens, mask, v)
    at = torch.arange(t)
    k = tokens.long().clamp(0, v - 1).unsqueeze(2)
    if placed:
        there = (tokens >= 0) & (tokens < v)
        first = torch.full((b, v), t).scatter_reduce_(1, k.squeeze(2), torch.where(there, at, t), "amin")
        z = z.masked_fill((first.unsqueeze(1) < at[:, None]).scatter(2, k, False), -math.inf)
    m = z.amax(2, keepdim=True)
    none = m == -math.inf
    e = torch.exp(z - torch.where(none, 0.0, m))
    own, others = e.gather(2, k), e.scatter(2, k, 0.0).sum(2, keepdim=True)
    total = torch.where(none, 1.0, others + own)
    lp = torch.where(others < own, -torch.log1p(others / own), (z.gather(2, k) - m) - torch.log(total))
    lp = torch.where(none, -math.inf, lp)
    ok = valid.unsqueeze(2)
    terms = min(v, max(4, v // 8 if v <= 64 else v // 64 + 64))
    return (torch.where(ok, e / total, 0.0), torch.where(ok, others / total, 0.0).squeeze(2), torch.where(ok, lp, 0.0).squeeze(2), valid,
            (1.5 * 40 + terms + 20) * U)
