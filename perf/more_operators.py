"""Operators around a learned order policy's products, as cases whose time is worth watching.

Between the layers of a policy stand a residual sum and a root-mean-square norm (cc_rms_norm), trained like the rest.  When
orders are sampled, products run on weights held in 8 bits: rows of activations are held in 8 bits too, with a scale each, by
the norm itself or by cc_quantize_rows, and cc_product_i8 multiplies the two.  The logits are then shaped (cc_shape_logits):
tokens that were there before are penalised or, as placed nodes are, forbidden, biases are added, and a grammar's mask leaves
out what may not follow.  A policy trained on the distribution that it samples from needs the gradient of that as well.

listed() names the cases, draw() gives others of the same ranges, prepare() makes what the program has in hand, run() is
one pass through one operator: the framework's calls where `own` is true, plain torch operations otherwise.  exact() is
the same from the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def listed():
    return [
        # Sampling: the state of 64 orders joins the residual stream and is normalised into 8 bits for the next product.
        {"name": "norm-step-q8", "kind": "norm", "rows": 64, "dim": 256, "dtype": "bf16", "weight": "f32", "residual": True, "form": "q8"},
        # Training: the positions of 1024 orders of 64 machines, a wide layer.
        {"name": "norm-n64-train", "kind": "norm", "rows": 65536, "dim": 1024, "dtype": "bf16", "weight": "f32", "residual": True, "form": "train"},
        # Training in 32 bits on five orders of a thousand machines; no second row starts where a vector load would like it.
        {"name": "norm-odd-train", "kind": "norm", "rows": 5000, "dim": 1021, "dtype": "f32", "weight": "f32", "residual": True, "form": "train"},
        # Sampling: the states of 1024 orders become rows of 8 bits.
        {"name": "quantize-step", "kind": "quantize", "rows": 1024, "dim": 128, "dtype": "f32"},
        # Loading: the table of a large odd vocabulary becomes channels of 8 bits.
        {"name": "quantize-vocab", "kind": "quantize", "rows": 50001, "dim": 1024, "dtype": "bf16"},
        # Sampling: logits over 64 machines for 1024 orders.
        {"name": "product-n64-step", "kind": "product", "rows": 1024, "channels": 64, "dim": 128, "dtype": "f32", "bias": True},
        # Sampling: logits of eight sequences over a large odd vocabulary; the weights are what there is to read.
        {"name": "product-vocab-step", "kind": "product", "rows": 8, "channels": 50001, "dim": 1024, "dtype": "bf16", "bias": False},
        # Scoring: odd in every size, no second row starts where a vector load would like it.
        {"name": "product-odd", "kind": "product", "rows": 777, "channels": 1001, "dim": 250, "dtype": "f16", "bias": True},
        # Scoring whole batches of long sequences through a wide layer: the matrix cores are what there is to fill.
        {"name": "product-large", "kind": "product", "rows": 8192, "channels": 8192, "dim": 4096, "dtype": "bf16", "bias": False},
        # Sampling orders of 64 machines: placed nodes are forbidden.
        {"name": "shape-n64-step", "kind": "shape", "batch": 1024, "length": 1, "vocab": 64, "history": 64, "dtype": "f32", "placed": True,
         "bias": False, "allowed": False, "train": False},
        # Sampling over a large vocabulary: prompts and what followed are penalised, a bias and a grammar hold.
        {"name": "shape-vocab-step", "kind": "shape", "batch": 128, "length": 1, "vocab": 131072, "history": 4096, "dtype": "bf16", "placed": False,
         "bias": True, "allowed": True, "train": False},
        # Training on orders of a thousand machines as they were sampled: at each rank the nodes placed before are forbidden.
        {"name": "shape-n1000-train", "kind": "shape", "batch": 64, "length": 1000, "vocab": 1000, "history": 1000, "dtype": "bf16", "placed": True,
         "bias": True, "allowed": False, "train": True},
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm", "quantize", "product", "product", "product", "shape", "shape", "shape"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("norm", "quantize"):
        dim = _log_between(rng, 16, 16384)
        case = {"kind": kind, "rows": _log_between(rng, 1, min(65536, (1 << 26) // dim)), "dim": dim, "dtype": dtype}
        if kind == "norm":
            case |= {"weight": rng.choice(["f32", dtype]), "residual": rng.random() < 0.75, "form": rng.choice(["train", "train", "plain", "q8"])}
        return case
    if kind == "product":
        dim, rows = _log_between(rng, 16, 8192), _log_between(rng, 1, 8192)
        most = min(65536, (1 << 26) // dim, (1 << 26) // rows, (1 << 37) // (rows * dim))
        return {"kind": kind, "rows": rows, "channels": _log_between(rng, 16, max(16, most)), "dim": dim, "dtype": dtype, "bias": rng.random() < 0.5}
    vocab = _log_between(rng, 8, 131072)
    placed = vocab <= 1024 and rng.random() < 0.6
    length = 1 if rng.random() < 0.4 else _log_between(rng, 2, vocab if placed else min(1024, (1 << 25) // vocab))
    batch = _log_between(rng, 1, min(4096, max(1, (1 << 25) // (vocab * length))))
    history = max(vocab, length) if placed else _log_between(rng, 1, min(8192, max(1, (1 << 22) // batch)))
    return {"kind": kind, "batch": batch, "length": length, "vocab": vocab, "history": history, "dtype": dtype, "placed": placed,
            "bias": rng.random() < 0.5, "allowed": rng.random() < 0.5, "train": rng.random() < 0.4}


# ---------------------------------------------------------------------------------------------------------- inputs


def _prepare_norm(case, g):
    n, d, dtype = case["rows"], case["dim"], DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    # what a layer adds is smaller than the stream that it joins; some channels are far larger than others
    loud = 1 + 9 * (torch.rand(d, generator=g, device="cuda") < 0.01)
    state = {"x": randn(n, d).to(dtype), "residual": None, "form": case["form"],
             "weight": (1 + 0.2 * randn(d)).to(DTYPES[case["weight"]])}
    if case["residual"]:
        state["residual"] = (3 * loud * randn(n, d)).to(dtype)
    if case["form"] == "train":
        state["grad"] = randn(n, d).to(dtype)
        state["grad_sum"] = randn(n, d).to(dtype) if case["residual"] else None
    return state


def _prepare_quantize(case, g):
    n, d = case["rows"], case["dim"]
    size = torch.exp(torch.randn(n, 1, generator=g, device="cuda"))
    return {"x": (size * torch.randn(n, d, generator=g, device="cuda")).to(DTYPES[case["dtype"]])}


def _prepare_product(case, g):
    m, n, k = case["rows"], case["channels"], case["dim"]

    def eight_bits(rows):
        # normal values whose largest in a row is some four deviations
        return (32 * torch.randn(rows, k, generator=g, device="cuda")).round_().clamp_(-127, 127).to(torch.int8)

    def scales(rows, size):
        return size * torch.exp(0.3 * torch.randn(rows, generator=g, device="cuda"))

    return {"x": eight_bits(m), "x_scale": scales(m, 1 / 32), "w": eight_bits(n), "w_scale": scales(n, 1 / (32 * math.sqrt(k))),
            "bias": torch.randn(n, generator=g, device="cuda") if case["bias"] else None, "dtype": DTYPES[case["dtype"]]}


def _prepare_shape(case, g):
    b, t, v, length, dtype = case["batch"], case["length"], case["vocab"], case["history"], DTYPES[case["dtype"]]

    def rand(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    state = {"logits": (3 * torch.randn(b, t, v, generator=g, device="cuda")).to(dtype), "starts": None, "bias": None, "allowed": None}
    if case["placed"]:
        # an order's nodes, each of them forbidden once it is placed; sampling has come to any rank
        order = rand(b, v).argsort(1).to(torch.int32)
        state["history"] = torch.full((b, length), -1, device="cuda", dtype=torch.int32)
        state["history"][:, :v] = order
        state["lengths"] = torch.randint(0, v - t + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        state["penalties"] = torch.tensor([1.0, math.inf, 0.0], device="cuda").expand(b, 3).contiguous()
    else:
        # tokens as unequally frequent as words are, a few of them padding; a part of each history is the prompt
        ids = (torch.exp(rand(b, length).double() * math.log(v + 1)) - 1).to(torch.int32).clamp_(0, v - 1)
        ids[rand(b, length) < 0.01] = -1
        state["history"] = ids
        state["lengths"] = (rand(b) * (max(0, length - t) + 1)).to(torch.int32)
        state["starts"] = (rand(b) * state["lengths"]).to(torch.int32)
        state["penalties"] = torch.stack([1 + 0.5 * rand(b), rand(b), 0.2 * rand(b)], 1)
    if case["bias"]:
        state["bias"] = torch.randn(v, generator=g, device="cuda")
    if case["allowed"]:
        words = torch.randint(-2**31, 2**31, (b, t, (v + 31) // 32), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        if b > 4:
            words[b // 2] = 0           # a grammar at its end allows nothing
        state["allowed"] = words
    if case["train"]:
        state["grad"] = torch.randn(b, t, v, generator=g, device="cuda").to(dtype)
    return state


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    state = {"norm": _prepare_norm, "quantize": _prepare_quantize, "product": _prepare_product, "shape": _prepare_shape}[kind](case, g)
    state["kind"] = kind
    return state


# ---------------------------------------------------------------------------------------------------- the framework


def _own_norm(state):
    import paper_2105_14088_amd as cc
    form = state["form"]
    res = cc.cc_rms_norm(state["x"], state["weight"], state["residual"], EPS, normed=form != "q8", quantized=form == "q8", save_rstd=form == "train")
    outputs = [] if state["residual"] is None else [res.sum]
    if form == "q8":
        return outputs + [res.q * res.scale.unsqueeze(1), res.scale]
    outputs.append(res.out)
    if form == "train":
        outputs += cc.cc_rms_norm_backward(state["grad"], res.sum, res.rstd, state["weight"], state["grad_sum"])
    return outputs


def _own_quantize(state):
    import paper_2105_14088_amd as cc
    q, scale = cc.cc_quantize_rows(state["x"])
    return [q * scale.unsqueeze(1), scale]


def _own_product(state):
    import paper_2105_14088_amd as cc
    return [cc.cc_product_i8(state["x"], state["x_scale"], state["w"], state["w_scale"], state["bias"], dtype=state["dtype"])]


def _own_shape(state):
    import paper_2105_14088_amd as cc
    args = (state["logits"], state["history"], state["lengths"], state["penalties"], state["starts"], state["bias"], state["allowed"])
    out = cc.cc_shape_logits(*args)
    if "grad" not in state:
        return [out]
    return [out, cc.cc_shape_logits_backward(state["grad"], *args)]


# ------------------------------------------------------------------------------------------------------- plain forms


def _eight_bits(u):
    """u [n, D] in 64 bits: whole numbers up to 127 and the largest of each row.  In 64 bits: which whole number is the nearest
    must not hang on a rounding."""
    most = u.abs().amax(1, keepdim=True)
    return torch.where(most > 0, torch.round(127 * u / most), 0.0), most


def _plain_norm(state):
    x, weight, dtype = state["x"], state["weight"].float(), state["x"].dtype
    h, outputs = x, []
    if state["residual"] is not None:
        h = (x.float() + state["residual"].float()).to(dtype)
        outputs = [h]
    wide = h.float()
    rstd = torch.rsqrt((wide * wide).mean(1, keepdim=True) + EPS)
    if state["form"] == "q8":
        q, most = _eight_bits(h.double() * state["weight"].double())
        scale = (most * rstd.double() / 127).float()
        return outputs + [q.float() * scale, scale.squeeze(1)]
    normed = wide * rstd
    outputs.append((normed * weight).to(dtype))
    if state["form"] == "train":
        grad = state["grad"].float()
        g = grad * weight
        grad_h = rstd * (g - normed * (g * normed).mean(1, keepdim=True))
        if state["grad_sum"] is not None:
            grad_h = grad_h + state["grad_sum"].float()
        outputs += [grad_h.to(dtype), (grad * normed).sum(0).to(state["weight"].dtype)]
    return outputs


def _plain_quantize(state):
    q, most = _eight_bits(state["x"].double())
    scale = (most / 127).float()
    return [q.float() * scale, scale.squeeze(1)]


def _plain_product(state):
    out = (state["x"].float() @ state["w"].float().t()) * state["x_scale"].unsqueeze(1) * state["w_scale"]
    if state["bias"] is not None:
        out = out + state["bias"]
    return [out.to(state["dtype"])]


def _plain_counts(state, since_start):
    """How often each token is among those that row t looks back on, [B, T, V] in whole numbers held in 32 bits."""
    history, lengths = state["history"], state["lengths"].unsqueeze(1)
    b, t, v = state["logits"].shape
    length = history.shape[1]
    at = torch.arange(length, device=history.device)
    real = (history >= 0) & (history < v)
    if since_start and state["starts"] is not None:
        real = real & (at >= state["starts"].unsqueeze(1))
    token = history.clamp(0, v - 1).long()
    # the row from which on a token is looked back on; what only later rows would see goes to a row that is cut off
    row = (at + 1 - lengths).clamp(min=0, max=t).long()
    counts = torch.zeros(b, (t + 1) * v, device=history.device).scatter_add_(1, row * v + token, real.float())
    return counts.view(b, t + 1, v)[:, :t].cumsum(1)


def _plain_forbidden(state, times):
    v = state["logits"].shape[2]
    presence, frequency = state["penalties"][:, 1, None, None], state["penalties"][:, 2, None, None]
    forbidden = (times > 0) & (torch.isposinf(presence) | torch.isposinf(frequency))
    if state["bias"] is not None:
        forbidden = forbidden | torch.isneginf(state["bias"])
    if state["allowed"] is not None:
        bits = (state["allowed"].unsqueeze(3) >> torch.arange(32, device=times.device, dtype=torch.int32)) & 1
        forbidden = forbidden | (bits.flatten(2)[:, :, :v] == 0)
    return forbidden


def _plain_shape(state):
    z, dtype = state["logits"].float(), state["logits"].dtype
    repetition, presence, frequency = (state["penalties"][:, i, None, None] for i in range(3))
    seen, times = _plain_counts(state, False) > 0, _plain_counts(state, True)
    forbidden = _plain_forbidden(state, times)
    out = torch.where(seen, torch.where(z > 0, z / repetition, z * repetition), z)
    out = torch.where(times > 0, out - presence - frequency * times, out)
    if state["bias"] is not None:
        out = out + state["bias"]
    out = torch.where(forbidden, -math.inf, out).to(dtype)
    if "grad" not in state:
        return [out]
    grad = state["grad"].float()
    grad = torch.where(seen, torch.where(z > 0, grad / repetition, grad * repetition), grad)
    return [out, torch.where(forbidden, 0.0, grad).to(dtype)]


def run(state):
    kind = state["kind"]
    if own:
        return {"norm": _own_norm, "quantize": _own_quantize, "product": _own_product, "shape": _own_shape}[kind](state)
    return {"norm": _plain_norm, "quantize": _plain_quantize, "product": _plain_product, "shape": _plain_shape}[kind](state)


# ---------------------------------------------------------------------------------------------------- in 64 bits


def _nearest_eighth(values, factor):
    """Rows of `values` as the nearest whole multiples of their largest / 127, times `factor`; and that step."""
    largest = torch.linalg.vector_norm(values, ord=math.inf, dim=1)
    safe = torch.where(largest == 0, 1.0, largest)
    steps = torch.round(values * 127 / safe[:, None])
    step = largest * factor / 127
    return steps * step[:, None], step


def _exact_norm(state):
    dtype = state["x"].dtype
    h = state["x"].double()
    outputs = []
    if state["residual"] is not None:
        # the sum is what the stream holds: an element of the type
        h = (h + state["residual"].double()).to(dtype).double()
        outputs.append(h)
    d = h.shape[1]
    w = state["weight"].double()
    s = 1 / torch.sqrt(torch.linalg.vector_norm(h, dim=1) ** 2 / d + EPS)
    if state["form"] == "q8":
        return outputs + list(_nearest_eighth(h * w, s))
    outputs.append(h * s[:, None] * w)
    if state["form"] == "train":
        dy = state["grad"].double()
        a = dy * w * s[:, None]
        along = (a * h).sum(1) * s * s / d
        dh = a - h * along[:, None]
        if state["grad_sum"] is not None:
            dh = dh + state["grad_sum"].double()
        outputs += [dh, s @ (dy * h)]
    return outputs


def _exact_product(state):
    x = state["x"].double() * state["x_scale"].double()[:, None]
    w = state["w"].double() * state["w_scale"].double()[:, None]
    out = torch.mm(x, w.t())
    return [out if state["bias"] is None else out + state["bias"].double()]


def _exact_shape(state):
    b, t, v = state["logits"].shape
    history, lengths = state["history"].long(), state["lengths"].tolist()
    starts = [0] * b if state["starts"] is None else state["starts"].tolist()
    out = torch.empty(b, t, v, device="cuda", dtype=torch.float64)
    grad = torch.empty_like(out) if "grad" in state else None
    r, p, f = (c.tolist() for c in state["penalties"].double().unbind(1))
    for i in range(b):
        # sequence by sequence: what each row looks back on, counted up to the first row and token by token from there
        first = lengths[i]
        before, later = history[i, :first], history[i, first:first + t - 1]
        new = torch.zeros(2, t, v, device="cuda", dtype=torch.float64)
        for which, since in ((0, 0), (1, starts[i])):
            kept = before[since:]
            new[which, 0] = torch.bincount(kept[(kept >= 0) & (kept < v)], minlength=v)[:v]
            rows = torch.arange(1, 1 + later.numel(), device="cuda")
            good = (later >= 0) & (later < v) & (first + rows - 1 >= since)
            new[which, rows[good], later[good]] += 1
        seen, times = new.cumsum(1)
        z = state["logits"][i].double()
        slope = torch.where(seen > 0, torch.where(z > 0, 1 / r[i], r[i]), 1.0)
        value = z * slope
        gone = torch.zeros_like(z, dtype=torch.bool)
        if math.isinf(p[i]) or math.isinf(f[i]):
            gone |= times > 0
        else:
            value = value - torch.where(times > 0, p[i] + f[i] * times, 0.0)
        if state["bias"] is not None:
            value = value + state["bias"].double()
        if state["allowed"] is not None:
            j = torch.arange(v, device="cuda")
            gone |= (state["allowed"][i].long()[:, j // 32] >> (j % 32)) & 1 == 0
        out[i] = value.masked_fill(gone, -math.inf)
        if grad is not None:
            grad[i] = (state["grad"][i].double() * slope).masked_fill(gone, 0.0)
    return [out] if grad is None else [out, grad]


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "quantize":
        return list(_nearest_eighth(state["x"].double(), 1.0))
    return {"norm": _exact_norm, "product": _exact_product, "shape": _exact_shape}[case["kind"]](state)


def work(case):
    """Bytes: inputs once, outputs once (rows in 8 bits as such, the history as the numbers that it is).  Operations: a sum, a
    square, a sum of squares and two products per normalised element, twice as many and a sum over rows where it is trained; a
    comparison, a product and a rounding per element brought to 8 bits; a product and a sum per term of a product; a
    comparison, a product and three sums per shaped logit, a comparison and a product where it has a gradient."""
    kind, e = case["kind"], BYTES[case["dtype"]]
    if kind in ("norm", "quantize"):
        n, d = case["rows"], case["dim"]
        if kind == "quantize":
            return {"bytes": n * d * (e + 1) + 4 * n, "flops": 3 * n * d}
        streams = 1 + 2 * case["residual"]                        # x, and the stream before and after
        nbytes, flops = streams * n * d * e + BYTES[case["weight"]] * d, 5 * n * d
        if case["form"] == "q8":
            return {"bytes": nbytes + n * d + 4 * n, "flops": flops + 3 * n * d}
        nbytes += n * d * e
        if case["form"] == "train":
            # the stream, the output's gradient and the stream's are read, one gradient is written
            nbytes, flops = nbytes + (3 + case["residual"]) * n * d * e + BYTES[case["weight"]] * d, flops + 10 * n * d
        return {"bytes": nbytes, "flops": flops}
    if kind == "product":
        m, n, k = case["rows"], case["channels"], case["dim"]
        return {"bytes": m * k + n * k + 4 * (m + n + n * case["bias"]) + m * n * e, "flops": 2 * m * n * k}
    rows = case["batch"] * case["length"]
    logits = rows * case["vocab"]
    nbytes = 2 * logits * e + 4 * case["batch"] * (case["history"] + 5) + 4 * case["vocab"] * case["bias"]
    if case["allowed"]:
        nbytes += 4 * rows * ((case["vocab"] + 31) // 32)
    if case["train"]:
        return {"bytes": nbytes + 3 * logits * e, "flops": 7 * logits}
    return {"bytes": nbytes, "flops": 5 * logits}
