"""The example that runs the order model's operators together: its gradient against automatic differentiation in 64 bits, and
what it learns."""
import importlib.util
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


def reference_logits(p, tokens, n, d, bias):
    """The policy's logits in 64 bits on the CPU, step by step."""
    b = tokens.shape[0]
    prev = torch.cat([torch.full((b, 1), n), tokens[:, :-1].long()], 1)
    x = p["nodes"][prev] + p["ranks"].unsqueeze(0)
    both = x @ p["mix"]
    h, hs = torch.zeros(b, d, dtype=torch.float64), []
    for t in range(n):
        keep = torch.sigmoid(both[:, t, d:] + bias)
        h = keep * h + (1 - keep) * both[:, t, :d]
        hs.append(h)
    return torch.stack(hs, 1) @ p["out"] + p["after"][prev]


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_the_whole_gradient(example, loss):
    """Every parameter's gradient is a chain of products in 32 bits whose longest sums have b n = 384 terms: each is off by no more than
    some 400 roundings (2^-24) of the sum of its terms' sizes, a few such sums follow each other; 1e-4 of the gradient's norm."""
    n, b = 24, 16
    policy = example.OrderPolicy(n, dim=20, seed=5)
    tokens = policy.sample(b, torch.Generator(device="cuda").manual_seed(2))
    assert all(sorted(r) == list(range(n)) for r in tokens.tolist())
    old = torch.full((b, n), -2.0, device="cuda")
    adv = torch.linspace(-1, 1, b, device="cuda")
    logits, saved = policy.forward(tokens)
    if loss == "policy":
        res = cc.cc_policy_loss(logits, tokens, old, adv, old, placed=True, kl_coef=0.05, clip_low=0.9, clip_high=50.0, mean="orders")
    else:
        res = cc.cc_preference_loss(logits, tokens, old, placed=True, beta=0.1)
    policy.backward(res.grad_logits, saved)

    p = {k: v.detach().cpu().double().requires_grad_(True) for k, v in policy.params.items()}
    z = reference_logits(p, tokens.cpu(), n, policy.dim, policy.gate_bias)
    want_logits = z.detach()
    gone = torch.zeros(b, n, n, dtype=torch.bool)
    for t in range(1, n):
        gone[:, t] = gone[:, t - 1].scatter(1, tokens[:, t - 1:t].cpu().long(), True)
    lp = torch.log_softmax(z.masked_fill(gone, float("-inf")), 2).gather(2, tokens.cpu().long().unsqueeze(2)).squeeze(2)
    if loss == "policy":
        r, a = torch.exp(lp + 2.0), adv.cpu().double().unsqueeze(1)
        kl = torch.exp(-2.0 - lp) - (-2.0 - lp) - 1
        value = (0.05 * kl - torch.minimum(r * a, r.clamp(0.1, 51.0) * a)).mean()
    else:
        gap = (lp + 2.0).sum(1)
        value = torch.nn.functional.softplus(-0.1 * (gap[:b // 2] - gap[b // 2:])).mean()
    value.backward()
    assert (logits.cpu().double() - want_logits).norm() <= 1e-5 * want_logits.norm()
    for k, v in policy.params.items():
        err = (v.grad.cpu().double() - p[k].grad).norm()
        assert err <= 1e-4 * p[k].grad.norm(), (k, float(err), float(p[k].grad.norm()))


@pytest.mark.parametrize("model,loss", [("tree", "policy"), ("bcube", "preference"), ("ring", "policy")])
def test_it_learns(example, model, loss):
    n, steps, batch = 16, 40, 256
    matrix = torch.from_numpy(random_matrix(n, 3, symmetric=True, lo=10, hi=2000)).cuda()
    best, cost, mean = example.learn(matrix, model, loss, steps=steps, batch=batch)
    assert sorted(best.tolist()) == list(range(n))
    assert int(example.score(model, matrix, best.view(1, -1))) == cost
    drawn = example.score(model, matrix, cc.cc_init_tours(n, steps * batch, 1)).double()
    assert mean < float(drawn.mean()) - 2 * float(drawn.std())           # the last batch is far from orders at random
