"""The operators of a learned order policy, as cases whose time is worth watching.

A policy over rank orders reads an order as a sequence of tokens: the nodes are the vocabulary, rank t is position t, and
a node that is placed is not placed again.  Its training step looks nodes up in a table (cc_embed), carries what has been
placed in a gated linear recurrence (cc_gated_scan), and learns from the costs of the orders it proposed, as advantages
(cc_policy_loss) or as pairs of a cheaper and a dearer order (cc_preference_loss); cc_token_logprob gives the
log-probabilities that these compare with.  The same calls serve sequences over any vocabulary.

listed() names the cases, draw() gives others of the same ranges, prepare() makes what the program has in hand, run() is
one pass through one operator: the framework's calls where `own` is true, plain torch operations otherwise.  exact() is
the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
CLIP_LOW, CLIP_HIGH, KL_COEF = 0.2, 0.28, 0.05
BETA, SMOOTHING = 0.1, 0.05


def listed():
    return [
        # Sampling: the last placed node of each of 1024 orders becomes a vector.
        {"name": "embed-n64-step", "kind": "embed", "vocab": 65, "tokens": 1024, "dim": 128, "dtype": "f32", "train": False},
        # Training on orders of a ragged thousand machines; the table has a row of its own for the start.
        {"name": "embed-n1000-train", "kind": "embed", "vocab": 1001, "tokens": 128000, "dim": 250, "dtype": "bf16", "train": True},
        # A large odd vocabulary whose tokens are as unequally frequent as words are.
        {"name": "embed-vocab-train", "kind": "embed", "vocab": 50001, "tokens": 65536, "dim": 1024, "dtype": "bf16", "train": True},
        # Sampling: one token more for 1024 orders, the state updated.
        {"name": "scan-step", "kind": "scan", "batch": 1024, "length": 1, "dim": 256, "dtype": "bf16", "train": False, "ragged": False},
        # Training on orders of 64 machines.
        {"name": "scan-n64-train", "kind": "scan", "batch": 1024, "length": 64, "dim": 128, "dtype": "f32", "train": True, "ragged": False},
        # Two long ragged sequences: the time axis is what there is to split.
        {"name": "scan-long-train", "kind": "scan", "batch": 2, "length": 65536, "dim": 1024, "dtype": "bf16", "train": True, "ragged": True},
        # Log-probabilities of 2048 orders of eight machines, as the reference policy gives them.
        {"name": "logprob-n8", "kind": "logprob", "batch": 2048, "length": 8, "vocab": 8, "dtype": "f32", "placed": True, "train": False},
        # Log-probabilities and their gradient under a loss of the user's own, 500 machines.
        {"name": "logprob-n500-train", "kind": "logprob", "batch": 128, "length": 500, "vocab": 500, "dtype": "f16", "placed": True, "train": True},
        # Policy step on a thousand orders of 64 machines.
        {"name": "policy-n64", "kind": "policy", "batch": 1024, "length": 64, "vocab": 64, "dtype": "f32", "placed": True, "mean": "tokens"},
        # Policy step on sequences over a large vocabulary.
        {"name": "policy-vocab", "kind": "policy", "batch": 16, "length": 512, "vocab": 65536, "dtype": "bf16", "placed": False, "mean": "orders"},
        # Preference step on pairs of orders of a thousand machines.
        {"name": "preference-n1000", "kind": "preference", "batch": 64, "length": 1000, "vocab": 1000, "dtype": "bf16", "placed": True},
        # Preference step on four pairs of sequences over an odd vocabulary: no row starts where a vector load would like it.
        {"name": "preference-vocab", "kind": "preference", "batch": 8, "length": 777, "vocab": 50001, "dtype": "f16", "placed": False},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["embed", "embed", "scan", "scan", "logprob", "policy", "policy", "preference", "preference"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind == "embed":
        dim = _log_between(rng, 16, 2048)
        return {"kind": kind, "vocab": _log_between(rng, 8, 100000), "tokens": _log_between(rng, 1, min(200000, (1 << 26) // dim)),
                "dim": dim, "dtype": dtype, "train": rng.random() < 0.75}
    if kind == "scan":
        dim = _log_between(rng, 16, 2048)
        length = 1 if rng.random() < 0.2 else _log_between(rng, 2, 65536)
        batch = _log_between(rng, 1, min(1024, max(1, (1 << 26) // (dim * length))))
        return {"kind": kind, "batch": batch, "length": length, "dim": dim, "dtype": dtype, "train": rng.random() < 0.75,
                "ragged": rng.random() < 0.5}
    placed = rng.random() < 0.6
    vocab = _log_between(rng, 8, 1024) if placed else _log_between(rng, 8, 131072)
    length = vocab if placed and rng.random() < 0.7 else _log_between(rng, 1, vocab if placed else 1024)
    batch = _log_between(rng, 1, min(4096, max(1, (1 << 27) // (vocab * length))))
    case = {"kind": kind, "batch": batch, "length": length, "vocab": vocab, "dtype": dtype, "placed": placed}
    if kind == "logprob":
        case["train"] = rng.random() < 0.5
    elif kind == "policy":
        case["mean"] = rng.choice(["tokens", "orders"])
    else:
        case["batch"] = 2 * max(1, batch // 2)
    return case


# ---------------------------------------------------------------------------------------------------------- inputs


def _prepare_embed(case, g):
    v, n, d, dtype = case["vocab"], case["tokens"], case["dim"], DTYPES[case["dtype"]]
    # nodes are equally frequent, words are not
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    ids = (u * v if v <= 1024 else torch.exp(u * math.log(v + 1)) - 1).to(torch.int32).clamp_(0, v - 1)
    # padding: a few tokens are no token
    ids[torch.rand(n, generator=g, device="cuda") < 0.01] = -1
    state = {"table": torch.randn(v, d, generator=g, device="cuda").to(dtype), "ids": ids, "scale": math.sqrt(d)}
    if case["train"]:
        state["grad"] = torch.randn(n, d, generator=g, device="cuda").to(dtype)
    return state


def _prepare_scan(case, g):
    b, t, d, dtype = case["batch"], case["length"], case["dim"], DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # value and gate lie side by side, as one product makes them; gates remember from two to some hundred steps
    both = torch.empty(b, t, 2 * d, device="cuda", dtype=dtype)
    for i in range(b):
        both[i, :, :d] = randn(t, d).to(dtype)
        both[i, :, d:] = (1.5 * randn(t, d) + 2).to(dtype)
    state = {"x": both[..., :d], "gate": both[..., d:], "h0": randn(b, d), "lengths": None}
    if case["ragged"]:
        lengths = torch.randint((t + 1) // 2, t + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        lengths[0] = t
        if b > 2:
            lengths[-1] = 0
        state["lengths"] = lengths
    if case["train"]:
        state["grad_h"] = torch.empty(b, t, d, device="cuda", dtype=dtype)
        for i in range(b):
            state["grad_h"][i] = randn(t, d).to(dtype)
        state["grad_last"] = randn(b, d)
    return state


def _token_state(case, g):
    b, t, v, dtype = case["batch"], case["length"], case["vocab"], DTYPES[case["dtype"]]
    logits = torch.empty(b, t, v, device="cuda", dtype=dtype)
    tokens = torch.empty(b, t, device="cuda", dtype=torch.int32)
    step = max(1, (1 << 26) // (t * v))
    for i in range(0, b, step):
        part = logits[i:i + step]
        z = 2 * torch.randn(part.shape, generator=g, device="cuda")
        part.copy_(z)
        if case["placed"]:
            # an order: its nodes in the sequence that a random priority gives
            tokens[i:i + step] = torch.rand(part.shape[0], v, generator=g, device="cuda").argsort(1)[:, :t]
        else:
            # a sample of the policy itself
            z += -torch.log(torch.empty_like(z).exponential_(generator=g))
            tokens[i:i + step] = z.argmax(2)
    # scored positions: a prefix is given, the tail is padding; one sequence of many has none that counts
    start = torch.randint(0, max(1, t // 8), (b, 1), generator=g, device="cuda")
    stop = t - torch.randint(0, max(1, t // 4), (b, 1), generator=g, device="cuda")
    at = torch.arange(t, device="cuda")
    mask = (at >= start) & (at < stop)
    if b > 4:
        mask[b // 2] = False
    return {"logits": logits, "tokens": tokens, "mask": mask, "placed": case["placed"], "scale": 0.75, "grad_scale": 1.0}


def _loss_scale(case, factor):
    """Half precision has five bits of exponent: a mean's gradient is scaled so that its terms lie among them."""
    return float(factor) if case["dtype"] == "f16" else 1.0


def _prepare_logprob(case, g):
    state = _token_state(case, g)
    if case["train"]:
        state["grad"] = torch.randn(case["batch"], case["length"], generator=g, device="cuda")
        state["grad_scale"] = _loss_scale(case, 256)
    return state


def _prepare_policy(case, g):
    state = _token_state(case, g)
    b, t = case["batch"], case["length"]
    now = _reference_logprob(state)
    # The policy has moved since it sampled: ratios about 1, some of them beyond the clip.  The gradient jumps where a
    # ratio meets the clip, so no ratio is left within one part in a thousand of it.
    ratio = torch.exp(0.25 * torch.randn(b, t, generator=g, device="cuda", dtype=torch.float64))
    for border in (1 - CLIP_LOW, 1 + CLIP_HIGH):
        near = (ratio / border - 1).abs() < 1e-3
        ratio = torch.where(near, ratio * 1.01, ratio)
    state["old"] = (now - torch.log(ratio)).to(torch.float32)
    state["ref"] = (now + 0.1 * torch.randn(b, t, generator=g, device="cuda")).to(torch.float32)
    # one advantage per order: its cost against the others'
    cost = torch.randn(b, generator=g, device="cuda")
    state["advantage"] = (cost.mean() - cost) / (cost.std() + 1e-6 if b > 1 else 1.0)
    state["mean"] = case["mean"]
    state["grad_scale"] = _loss_scale(case, 64 * b * t)
    return state


def _prepare_preference(case, g):
    state = _token_state(case, g)
    b, t = case["batch"], case["length"]
    # the policy has begun to prefer the first of each pair: some five nats a sequence, however long it is
    ahead = torch.full((b, 1), 5 / t, device="cuda", dtype=torch.float64)
    ahead[b // 2:] *= -1
    state["ref"] = (_reference_logprob(state) - ahead + 0.1 * torch.randn(b, t, generator=g, device="cuda")).to(torch.float32)
    state["grad_scale"] = _loss_scale(case, 4096 * (b // 2))
    return state


def _reference_logprob(state):
    """Log-probabilities in 64 bits, as another copy of the policy would have given them."""
    b, t, v = state["logits"].shape
    out = torch.zeros(b, t, device="cuda", dtype=torch.float64)
    step = max(1, (1 << 25) // (t * v))
    for i in range(0, b, step):
        z = state["logits"][i:i + step].to(torch.float64) * state["scale"]
        token = state["tokens"][i:i + step].long().unsqueeze(2)
        if state["placed"]:
            z = z.masked_fill(_placed(state["tokens"][i:i + step], v), -math.inf)
        out[i:i + step] = z.gather(2, token).squeeze(2) - torch.logsumexp(z, 2)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    state = {"embed": _prepare_embed, "scan": _prepare_scan, "logprob": _prepare_logprob, "policy": _prepare_policy,
             "preference": _prepare_preference}[kind](case, g)
    state["kind"] = kind
    return state


# ---------------------------------------------------------------------------------------------------- the framework


def _own_embed(state):
    import paper_2105_14088_amd as cc
    out = cc.cc_embed(state["table"], state["ids"], state["scale"])
    if "grad" not in state:
        return [out]
    return [out, cc.cc_embed_backward(state["grad"], state["ids"], state["table"].shape[0], state["scale"])]


def _own_scan(state):
    import paper_2105_14088_amd as cc
    train = "grad_h" in state
    h, last, states = cc.cc_gated_scan(state["x"], state["gate"], state["h0"], state["lengths"], save_states=train)
    if not train:
        return [h, last]
    return [h, last, *cc.cc_gated_scan_backward(state["x"], state["gate"], states, state["grad_h"], state["grad_last"], state["lengths"])]


def _own_logprob(state):
    import paper_2105_14088_amd as cc
    args = (state["logits"], state["tokens"], state["mask"], state["placed"], state["scale"])
    logprob, rows = cc.cc_token_logprob(*args)
    if "grad" not in state:
        return [logprob]
    return [logprob, cc.cc_token_logprob_backward(*args, rows, state["grad"], grad_scale=state["grad_scale"])]


def _own_policy(state):
    import paper_2105_14088_amd as cc
    res = cc.cc_policy_loss(state["logits"], state["tokens"], state["old"], state["advantage"], state["ref"], state["mask"],
                            placed=state["placed"], scale=state["scale"], clip_low=CLIP_LOW, clip_high=CLIP_HIGH,
                            kl_coef=KL_COEF, mean=state["mean"], grad_scale=state["grad_scale"])
    return [res.stats, res.logprob, res.grad_logits]


def _own_preference(state):
    import paper_2105_14088_amd as cc
    res = cc.cc_preference_loss(state["logits"], state["tokens"], state["ref"], state["mask"], placed=state["placed"],
                                scale=state["scale"], beta=BETA, label_smoothing=SMOOTHING, grad_scale=state["grad_scale"])
    return [res.loss, res.margin, res.logprob, res.grad_logits]


# ------------------------------------------------------------------------------------------------------- plain forms


def _plain_embed(state):
    table, ids = state["table"], state["ids"]
    v, d = table.shape
    valid = ((ids >= 0) & (ids < v)).unsqueeze(1)
    index = ids.clamp(0, v - 1).long()
    out = torch.where(valid, table[index].float() * state["scale"], 0.0).to(table.dtype)
    if "grad" not in state:
        return [out]
    rows = torch.where(valid, state["grad"].float() * state["scale"], 0.0)
    return [out, torch.zeros(v, d, device=table.device).index_add_(0, index, rows).to(table.dtype)]


def _doubling_scan(a, b):
    """h_t = a_t h_{t-1} + b_t along axis 1: after k steps an element has taken in the 2^k before it."""
    t, step = a.shape[1], 1
    while step < t:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        if 2 * step < t:
            a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return b


def _plain_scan(state):
    x, gate, h0, dtype = state["x"].float(), state["gate"].float(), state["h0"], state["x"].dtype
    t = x.shape[1]
    a, c = torch.sigmoid(gate), torch.sigmoid(-gate)
    b = c * x
    inside = None
    if state["lengths"] is not None:
        inside = (torch.arange(t, device=x.device) < state["lengths"].unsqueeze(1)).unsqueeze(2)
        a, b = torch.where(inside, a, 1.0), torch.where(inside, b, 0.0)
    b = torch.cat([b[:, :1] + a[:, :1] * h0.unsqueeze(1), b[:, 1:]], 1)
    h = _doubling_scan(a, b)
    last = h[:, -1].clone()
    out = (h if inside is None else torch.where(inside, h, 0.0)).to(dtype)
    if "grad_h" not in state:
        return [out, last]
    grad = state["grad_h"].float()
    if inside is not None:
        grad = torch.where(inside, grad, 0.0)
    grad = torch.cat([grad[:, :-1], grad[:, -1:] + state["grad_last"].unsqueeze(1)], 1)
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    lam = _doubling_scan(after.flip(1), grad.flip(1)).flip(1)
    before = torch.cat([h0.unsqueeze(1), h[:, :-1]], 1)
    dx, dgate = c * lam, lam * (before - x) * (a * c)
    if inside is not None:
        dx, dgate = torch.where(inside, dx, 0.0), torch.where(inside, dgate, 0.0)
    return [out, last, dx.to(dtype), dgate.to(dtype), a[:, 0] * lam[:, 0]]


def _placed(tokens, v):
    """[B, T, V]: the node went to an earlier rank, and is not the one at this rank."""
    b, t = tokens.shape
    at = torch.arange(t, device=tokens.device)
    first = torch.full((b, v), t, device=tokens.device, dtype=torch.int64)
    first.scatter_reduce_(1, tokens.long(), at.expand(b, t), "amin")
    return first.unsqueeze(1) < at[:, None]


def _plain_row_terms(state):
    """Candidates' exponentials, their sum without the token's own, the sum, log-probability and what counts."""
    logits, tokens = state["logits"], state["tokens"]
    v = logits.shape[2]
    z = logits.float() * state["scale"]
    token = tokens.long().unsqueeze(2)
    if state["placed"]:
        z = z.masked_fill(_placed(tokens, v), -math.inf)
    z = z - z.amax(2, keepdim=True)
    chosen = z.gather(2, token)
    e = torch.exp(z)
    others = e.scatter(2, token, 0.0).sum(2, keepdim=True)
    total = others + torch.exp(chosen)
    # long sums of log-probabilities are compared with each other: they are held in 64 bits
    wide = chosen.double()
    logprob = torch.where(wide == 0, -torch.log1p(others.double()), wide - torch.log(others.double() + torch.exp(wide)))
    return e, others, total, torch.where(state["mask"], logprob.squeeze(2), 0.0)


def _plain_grad_logits(state, e, others, total, slope):
    """slope: d loss / d logprob [B, T]."""
    s = (state["scale"] * state["grad_scale"] * torch.where(state["mask"], slope, 0.0)).unsqueeze(2)
    grad = (-s / total) * e
    grad.scatter_(2, state["tokens"].long().unsqueeze(2), s * others / total)
    return torch.where(state["mask"].unsqueeze(2), grad, 0.0).to(state["logits"].dtype)


def _plain_logprob(state):
    e, others, total, logprob = _plain_row_terms(state)
    if "grad" not in state:
        return [logprob.float()]
    return [logprob.float(), _plain_grad_logits(state, e, others, total, state["grad"])]


def _plain_policy(state):
    e, others, total, logprob = _plain_row_terms(state)
    mask = state["mask"]
    count = mask.sum(1, keepdim=True)
    if state["mean"] == "tokens":
        weight = mask.float() / count.sum().clamp(min=1)
    else:
        weight = mask.float() / count.clamp(min=1) / (count > 0).sum().clamp(min=1)
    advantage = state["advantage"].unsqueeze(1)
    ratio = torch.exp(logprob - state["old"]).float()
    free, held = ratio * advantage, ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH) * advantage
    clipped = held < free
    away = state["ref"] - logprob
    kl = (torch.expm1(away) - away).float()
    terms = torch.stack([KL_COEF * kl - torch.minimum(free, held), kl, clipped.float()])
    stats = torch.where(mask, terms * weight, 0.0).sum((1, 2), dtype=torch.float64).to(torch.float32)
    slope = weight * (-KL_COEF * torch.expm1(away).float() - torch.where(clipped, 0.0, free))
    return [stats, logprob.float(), _plain_grad_logits(state, e, others, total, slope)]


def _plain_preference(state):
    e, others, total, logprob = _plain_row_terms(state)
    pairs = logprob.shape[0] // 2
    gap = torch.where(state["mask"], logprob - state["ref"], 0.0).sum(1)
    margin = BETA * (gap[:pairs] - gap[pairs:])
    loss = (1 - SMOOTHING) * torch.log1p(torch.exp(-margin.abs())) + (1 - SMOOTHING) * (-margin).clamp(min=0)
    loss = loss + SMOOTHING * torch.log1p(torch.exp(-margin.abs())) + SMOOTHING * margin.clamp(min=0)
    slope = (BETA / pairs * (torch.sigmoid(margin) - (1 - SMOOTHING))).float()
    slope = torch.cat([slope, -slope]).unsqueeze(1).expand_as(logprob)
    return [loss.mean().float(), margin.float(), logprob.float(), _plain_grad_logits(state, e, others, total, slope)]


def run(state):
    kind = state["kind"]
    if own:
        return {"embed": _own_embed, "scan": _own_scan, "logprob": _own_logprob, "policy": _own_policy,
                "preference": _own_preference}[kind](state)
    return {"embed": _plain_embed, "scan": _plain_scan, "logprob": _plain_logprob, "policy": _plain_policy,
            "preference": _plain_preference}[kind](state)


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _exact_embed(state):
    table, ids = state["table"].double(), state["ids"].long()
    out = torch.zeros(ids.numel(), table.shape[1], device="cuda", dtype=torch.float64)
    real = (ids >= 0).nonzero().squeeze(1)
    out[real] = table[ids[real]] * state["scale"]
    if "grad" not in state:
        return [out]
    # tokens in order of their id, a sum for each run of one id
    order = real[ids[real].argsort(stable=True)]
    counts = torch.bincount(ids[real], minlength=table.shape[0]).cpu().tolist()
    grad = torch.zeros_like(table)
    at = 0
    rows = state["grad"]
    for v, n in enumerate(counts):
        if n:
            grad[v] = rows[order[at:at + n]].double().sum(0) * state["scale"]
            at += n
    return [out, grad]


def _exact_scan(state):
    value, gate, h0 = state["x"].double(), state["gate"].double(), state["h0"].double()
    b, t, d = value.shape
    inside = torch.ones(b, t, 1, device="cuda", dtype=torch.bool)
    if state["lengths"] is not None:
        inside = (torch.arange(t, device="cuda") < state["lengths"].unsqueeze(1)).unsqueeze(2)
    # step by step; beyond its length a sequence keeps its state
    keep = torch.where(inside, 1 / (1 + torch.exp(-gate)), 1.0)
    take = torch.where(inside, 1 / (1 + torch.exp(gate)), 0.0)
    hs, s = take * value, h0
    for i in range(t):
        s = torch.addcmul(hs[:, i], keep[:, i], s)
        hs[:, i] = s
    h = torch.where(inside, hs, 0.0)
    if "grad_h" not in state:
        return [h, s]
    lam, flow = torch.where(inside, state["grad_h"].double(), 0.0), state["grad_last"].double()
    for i in range(t - 1, -1, -1):
        flow = flow + lam[:, i]
        lam[:, i] = flow
        flow = flow * keep[:, i]
    before = torch.cat([h0.unsqueeze(1), hs[:, :-1]], 1)
    return [h, s, take * lam, torch.where(inside, lam * (before - value) * keep * take, 0.0), flow]


def _exact_rows(state, i, j):
    """Probabilities, their complement at the token and log-probabilities of orders i .. j-1."""
    z = state["logits"][i:j].double() * state["scale"]
    tokens = state["tokens"][i:j].long()
    if state["placed"]:
        hot = torch.nn.functional.one_hot(tokens, z.shape[2]).bool()
        gone = (hot.cumsum(1) - hot.long() > 0) & ~hot
        z = torch.where(gone, -math.inf, z)
    lse = torch.logsumexp(z, 2, keepdim=True)
    p = torch.exp(z - lse)
    chosen = tokens.unsqueeze(2)
    rest = p.scatter(2, chosen, 0.0).sum(2)
    logprob = torch.where(rest < 0.5, torch.log1p(-rest), (z.gather(2, chosen) - lse).squeeze(2))
    return p, rest, logprob, chosen


def _exact_pieces(state, slope_of):
    """Log-probabilities, and the logits' gradient once slope_of(log-probabilities) is known."""
    b, t, v = state["logits"].shape
    step = max(1, (1 << 25) // (t * v))
    logprob = torch.cat([_exact_rows(state, i, min(b, i + step))[2] for i in range(0, b, step)])
    logprob = torch.where(state["mask"], logprob, 0.0)
    if slope_of is None:
        return logprob, None
    slope = torch.where(state["mask"], slope_of(logprob), 0.0) * state["scale"] * state["grad_scale"]
    grad = torch.empty(b, t, v, device="cuda", dtype=torch.float64)
    for i in range(0, b, step):
        j = min(b, i + step)
        p, rest, _, chosen = _exact_rows(state, i, j)
        s = slope[i:j].unsqueeze(2)
        grad[i:j] = (p * -s).scatter(2, chosen, s * rest.unsqueeze(2))
    return logprob, grad


def _exact_logprob(state):
    if "grad" not in state:
        return [_exact_pieces(state, None)[0]]
    return list(_exact_pieces(state, lambda lp: state["grad"].double()))


def _exact_policy(state):
    mask = state["mask"].double()
    per_order = mask.sum(1)
    if state["mean"] == "tokens":
        weight = mask / max(1.0, float(mask.sum()))
    else:
        weight = mask / per_order.clamp(min=1).unsqueeze(1) / max(1, int((per_order > 0).sum()))
    adv, old, ref = state["advantage"].double().unsqueeze(1), state["old"].double(), state["ref"].double()
    found = {}

    def slope_of(lp):
        r = torch.exp(lp - old)
        # a gain beyond the upper border, or a loss below the lower one, no longer pulls
        beyond = ((adv > 0) & (r > 1 + CLIP_HIGH)) | ((adv < 0) & (r < 1 - CLIP_LOW))
        kl = torch.expm1(ref - lp) - (ref - lp)
        gain = torch.where(beyond, torch.where(adv > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW) * adv, r * adv)
        found["stats"] = torch.stack([(weight * (KL_COEF * kl - gain)).sum(), (weight * kl).sum(), (weight * beyond).sum()])
        return weight * (-KL_COEF * torch.expm1(ref - lp) - torch.where(beyond, 0.0, r * adv))

    logprob, grad = _exact_pieces(state, slope_of)
    return [found["stats"], logprob, grad]


def _exact_preference(state):
    found = {}

    def slope_of(lp):
        pairs = lp.shape[0] // 2
        gap = ((lp - state["ref"].double()) * state["mask"]).sum(1)
        m = BETA * (gap[:pairs] - gap[pairs:])
        zero = torch.zeros_like(m)
        found["loss"] = ((1 - SMOOTHING) * torch.logaddexp(zero, -m) + SMOOTHING * torch.logaddexp(zero, m)).mean()
        found["margin"] = m
        pull = BETA / pairs * (SMOOTHING / (1 + torch.exp(-m)) - (1 - SMOOTHING) / (1 + torch.exp(m)))
        return torch.cat([pull, -pull]).unsqueeze(1).expand_as(lp)

    logprob, grad = _exact_pieces(state, slope_of)
    return [found["loss"], found["margin"], logprob, grad]


def exact(case, seed):
    state = prepare(case, seed)
    return {"embed": _exact_embed, "scan": _exact_scan, "logprob": _exact_logprob, "policy": _exact_policy,
            "preference": _exact_preference}[case["kind"]](state)


def work(case):
    """Bytes: inputs once, outputs once (the rows of a table that are looked up, at most one per token).  Operations: a
    multiply per looked-up and an add per summed element; a sigmoid, a product and a sum per element and step; a
    scaling, an exponential and a sum per logit, and a product where it has a gradient."""
    e = BYTES[case["dtype"]]
    if case["kind"] == "embed":
        v, n, d = case["vocab"], case["tokens"], case["dim"]
        nbytes = min(n, v) * d * e + 4 * n + n * d * e
        if not case["train"]:
            return {"bytes": nbytes, "flops": n * d}
        return {"bytes": nbytes + n * d * e + v * d * e, "flops": 3 * n * d}
    if case["kind"] == "scan":
        rows = case["batch"] * case["length"] * case["dim"]
        ends = 4 * case["batch"] * case["dim"]
        nbytes, flops = 3 * rows * e + 2 * ends, 8 * rows
        if case["train"]:
            nbytes, flops = nbytes + 3 * rows * e + 2 * ends, flops + 12 * rows
        return {"bytes": nbytes, "flops": flops}
    rows = case["batch"] * case["length"]
    logits = rows * case["vocab"]
    nbytes, flops = logits * e + rows * 9, 4 * logits
    if case["kind"] != "logprob" or case["train"]:
        nbytes, flops = nbytes + logits * e + rows * 8, flops + 2 * logits
    return {"bytes": nbytes, "flops": flops}
