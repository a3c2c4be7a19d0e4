"""The example with the norm, products in 8 bits and shaped logits: its gradient against automatic differentiation in 64 bits, its sampling
against the same by torch's operations, and that it runs."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2105_14088_amd as cc
from gen import random_matrix

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("learn_order", os.path.join(ROOT, "examples", "learn_order.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference_logits(p, tokens, policy):
    """The policy's logits in 64 bits on the CPU, step by step."""
    n, d, b = policy.n, policy.dim, tokens.shape[0]
    prev = torch.cat([torch.full((b, 1), n), tokens[:, :-1].long()], 1)
    stream = p["nodes"][prev] + p["ranks"].unsqueeze(0)
    h = None
    for i in range(policy.layers):
        y = stream
        if i:
            stream = stream + h
            y = stream / torch.sqrt((stream * stream).mean(2, keepdim=True) + 1e-6) * p[f"norm{i}"]
        both = y @ p[f"mix{i}" if i else "mix"]
        state, hs = torch.zeros(b, d, dtype=torch.float64), []
        for t in range(n):
            keep = torch.sigmoid(both[:, t, d:] + policy.gate_bias)
            state = keep * state + (1 - keep) * both[:, t, :d]
            hs.append(state)
        h = torch.stack(hs, 1)
    return h @ p["out"] + p["after"][prev]


@pytest.mark.parametrize("layers", [1, 2, 3])
def test_the_whole_gradient(example, layers):
    """As for the policy of one layer: chains of sums of at most some 400 terms in 32 bits, 400 * 2^-24 = 2.4e-5 of the sum of the terms' sizes
    each, three of them for a layer; 3e-4 of the gradient's norm for three layers."""
    n, b = 20, 16
    policy = example.OrderPolicy(n, dim=24, seed=3, layers=layers)
    g = torch.Generator(device="cuda").manual_seed(9)
    for name, p in policy.params.items():
        if name.startswith("norm"):
            p += 0.2 * torch.randn(p.shape, generator=g, device="cuda")
    tokens = policy.sample(b, torch.Generator(device="cuda").manual_seed(2))
    assert all(sorted(r) == list(range(n)) for r in tokens.tolist())
    logits, saved = policy.forward(tokens)
    weight = torch.randn(b, n, generator=g, device="cuda")
    lp, rows = cc.cc_token_logprob(logits, tokens, placed=True)
    policy.backward(cc.cc_token_logprob_backward(logits, tokens, None, True, 1.0, rows, weight), saved)

    p = {k: v.detach().cpu().double().requires_grad_(True) for k, v in policy.params.items()}
    z = reference_logits(p, tokens.cpu(), policy)
    gone = torch.zeros(b, n, n, dtype=torch.bool)
    for t in range(1, n):
        gone[:, t] = gone[:, t - 1].scatter(1, tokens[:, t - 1:t].cpu().long(), True)
    want = torch.log_softmax(z.masked_fill(gone, -math.inf), 2).gather(2, tokens.cpu().long().unsqueeze(2)).squeeze(2)
    (want * weight.cpu().double()).sum().backward()
    assert (logits.cpu().double() - z.detach()).norm() <= 1e-5 * layers * z.detach().norm()
    for k, v in policy.params.items():
        err = (v.grad.cpu().double() - p[k].grad).norm()
        assert err <= 1e-4 * layers * p[k].grad.norm(), (k, float(err), float(p[k].grad.norm()))


def test_sampling_is_what_masking_gave(example):
    """The placed nodes' logits filled with minus infinity by torch: the same orders, bit for bit."""
    n, count = 48, 300
    policy = example.OrderPolicy(n, seed=4)
    p, d = policy.params, policy.dim
    g = torch.Generator(device="cuda").manual_seed(8)
    want = torch.empty(count, n, dtype=torch.int32, device="cuda")
    state = torch.zeros(count, d, device="cuda")
    prev = torch.full((count, 1), n, dtype=torch.int32, device="cuda")
    placed = torch.zeros(count, n, dtype=torch.bool, device="cuda")
    for t in range(n):
        both = (cc.cc_embed(p["nodes"], prev) + cc.cc_embed(p["ranks"], torch.full_like(prev, t))) @ p["mix"]
        both[..., d:] += policy.gate_bias
        h, _, _ = cc.cc_gated_scan(both[..., :d], both[..., d:], state, last=state)
        logits = (h @ p["out"] + cc.cc_embed(p["after"], prev))[:, 0]
        noise = -torch.log(torch.empty_like(logits).exponential_(generator=g))
        prev = (logits + noise).masked_fill_(placed, -math.inf).argmax(1, keepdim=True).to(torch.int32)
        placed.scatter_(1, prev.long(), True)
        want[:, t:t + 1] = prev
    assert torch.equal(policy.sample(count, torch.Generator(device="cuda").manual_seed(8)), want)


@pytest.mark.parametrize("layers", [1, 2])
def test_sampling_in_8_bits(example, layers):
    n, count = 33, 200
    policy = example.OrderPolicy(n, dim=40, seed=6, layers=layers)
    orders = policy.sample(count, torch.Generator(device="cuda").manual_seed(1), bits=8)
    assert (orders.sort(1).values == torch.arange(n, device="cuda")).all()


def test_it_runs(example):
    matrix = torch.from_numpy(random_matrix(16, 3, symmetric=True, lo=10, hi=2000)).cuda()
    best, cost, _ = example.learn(matrix, "bcube", steps=3, batch=64, layers=2, bits=8)
    assert sorted(best.tolist()) == list(range(16)) and int(example.score("bcube", matrix, best.view(1, -1))) == cost
