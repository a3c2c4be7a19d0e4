"""A rank order learnt from costs: for models that have a batch call and no search (double binary tree, BCube), or any other
that a batch of orders can be scored by.

A small policy proposes orders node by node: the node placed last and the rank to fill are looked up (cc_embed), a gated
recurrence carries what has been placed (cc_gated_scan), one product makes logits, nodes that are placed are left out.  The
orders are scored by the library's batch call; the cheaper ones are made more probable, by the clipped policy loss on
advantages (cc_policy_loss) or by the preference loss on pairs of a cheaper and a dearer order (cc_preference_loss).
Sampling runs the same calls a token at a time.  Products and the optimiser are torch's.

    python examples/learn_order.py --model tree --steps 200
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2105_14088_amd as cc  # noqa: E402
from gen import make_matrix, random_matrix  # noqa: E402


class OrderPolicy:
    def __init__(self, n: int, dim: int = 64, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def new(*shape, scale):
            return (scale * torch.randn(*shape, generator=g, device="cuda")).requires_grad_(False)

        self.n, self.dim = n, dim
        self.params = {
            "nodes": new(n + 1, dim, scale=1.0),                # row n: nothing placed yet
            "ranks": new(n, dim, scale=1.0),
            "after": new(n + 1, n, scale=0.01),                 # logits of a node by the one before it
            "mix": new(dim, 2 * dim, scale=1 / math.sqrt(dim)),  # values and gates in one product
            "out": new(dim, n, scale=0.1 / math.sqrt(dim)),
        }
        for p in self.params.values():
            p.grad = torch.zeros_like(p)
        self.gate_bias = 2.0

    def _mixed(self, prev, ranks):
        """Values and gates [B, T, dim] of what was placed last and the rank to fill, and their sum's two parts' input."""
        p = self.params
        x = cc.cc_embed(p["nodes"], prev) + cc.cc_embed(p["ranks"], ranks)
        both = x @ p["mix"]
        both[..., self.dim:] += self.gate_bias
        return x, both[..., :self.dim], both[..., self.dim:]

    def sample(self, count: int, generator) -> torch.Tensor:
        """`count` orders, int32 [count, n]: a token at a time, the state updated in place."""
        p, n = self.params, self.n
        tokens = torch.empty(count, n, dtype=torch.int32, device="cuda")
        state = torch.zeros(count, self.dim, device="cuda")
        prev = torch.full((count, 1), n, dtype=torch.int32, device="cuda")
        placed = torch.zeros(count, n, dtype=torch.bool, device="cuda")
        for t in range(n):
            rank = torch.full_like(prev, t)
            _, value, gate = self._mixed(prev, rank)
            h, _, _ = cc.cc_gated_scan(value, gate, state, last=state)
            logits = (h @ p["out"] + cc.cc_embed(p["after"], prev))[:, 0]
            noise = -torch.log(torch.empty_like(logits).exponential_(generator=generator))
            prev = (logits + noise).masked_fill_(placed, -math.inf).argmax(1, keepdim=True).to(torch.int32)
            placed.scatter_(1, prev.long(), True)
            tokens[:, t:t + 1] = prev
        return tokens

    def forward(self, tokens):
        b, n = tokens.shape
        p = self.params
        prev = torch.cat([torch.full_like(tokens[:, :1], n), tokens[:, :-1]], 1).contiguous()
        ranks = torch.arange(n, dtype=torch.int32, device="cuda").expand(b, n).contiguous()
        x, value, gate = self._mixed(prev, ranks)
        h, _, states = cc.cc_gated_scan(value, gate, save_states=True)
        logits = h @ p["out"] + cc.cc_embed(p["after"], prev)
        return logits, (prev, ranks, x, value, gate, h, states)

    def backward(self, grad_logits, saved):
        """Adds the parameters' gradients to what is there."""
        prev, ranks, x, value, gate, h, states = saved
        p, n, d = self.params, self.n, self.dim
        flat = grad_logits.reshape(-1, n)
        p["out"].grad += h.reshape(-1, d).t() @ flat
        cc.cc_embed_backward(grad_logits, prev, n + 1, grad_table=p["after"].grad, accumulate=True)
        both = torch.empty(*h.shape[:2], 2 * d, device="cuda")
        cc.cc_gated_scan_backward(value, gate, states, (flat @ p["out"].t()).view_as(h), grad_x=both[..., :d], grad_gate=both[..., d:])
        both = both.view(-1, 2 * d)
        p["mix"].grad += x.reshape(-1, d).t() @ both
        grad_x = (both @ p["mix"].t()).view_as(x)
        cc.cc_embed_backward(grad_x, prev, n + 1, grad_table=p["nodes"].grad, accumulate=True)
        cc.cc_embed_backward(grad_x, ranks, n, grad_table=p["ranks"].grad, accumulate=True)


def score(model: str, matrix: torch.Tensor, orders: torch.Tensor) -> torch.Tensor:
    if model == "tree":
        return cc.cc_dbt_cost_batch(matrix, orders)
    if model == "bcube":
        return cc.cc_bcube_cost_batch(matrix, 4, orders)
    return cc.cc_ring_cost_batch(matrix, orders, cc.CC_RING_SUM)


def learn(matrix: torch.Tensor, model: str, loss: str = "policy", steps: int = 200, batch: int = 1024, rounds: int = 3,
          rate: float = 0.015, seed: int = 1, say=lambda *a: None):
    """(best order, its cost, mean cost of the last batch)."""
    n = matrix.shape[0]
    policy = OrderPolicy(n, seed=seed)
    optimiser = torch.optim.Adam(policy.params.values(), lr=rate)
    g = torch.Generator(device="cuda").manual_seed(seed)
    best_cost, best = None, None
    for step in range(steps):
        for group in optimiser.param_groups:
            group["lr"] = rate * (1 - step / steps)
        orders = policy.sample(batch, g)
        cost = score(model, matrix, orders)
        low, at = cost.min(0)
        if best_cost is None or int(low) < best_cost:
            best_cost, best = int(low), orders[at].clone()
        advantage = -(cost - cost.double().mean()).double()
        advantage = (advantage / (advantage.std() + 1e-9)).float()
        if loss == "preference":
            # the cheaper half, cheapest first, against the dearer half
            orders = orders[cost.argsort()].contiguous()
        logits, _ = policy.forward(orders)
        old, _ = cc.cc_token_logprob(logits, orders, placed=True)
        for _ in range(rounds):
            logits, saved = policy.forward(orders)
            if loss == "preference":
                res = cc.cc_preference_loss(logits, orders, old, placed=True, beta=0.1, grad_logits=logits)
            else:
                res = cc.cc_policy_loss(logits, orders, old, advantage, old, placed=True, kl_coef=0.05, mean="orders", grad_logits=logits)
            optimiser.zero_grad(set_to_none=False)
            policy.backward(res.grad_logits, saved)
            optimiser.step()
        if step % 20 == 0 or step == steps - 1:
            say(f"step {step:4d}: mean cost {float(cost.double().mean()):.0f}, best so far {best_cost}")
    return best, best_cost, float(cost.double().mean())


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--model", choices=["tree", "bcube", "ring"], default="tree")
    ap.add_argument("--loss", choices=["policy", "preference"], default="policy")
    ap.add_argument("--n", type=int, default=64, help="64: the synthetic 64-node matrix; else a random symmetric one")
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--batch", type=int, default=1024)
    ap.add_argument("--seed", type=int, default=1)
    args = ap.parse_args()
    host = make_matrix(2) if args.n == 64 else random_matrix(args.n, 7, symmetric=True, lo=10, hi=2000)
    matrix = torch.from_numpy(host).cuda()
    best, cost, _ = learn(matrix, args.model, args.loss, args.steps, args.batch, seed=args.seed, say=lambda s: print(s, flush=True))
    assert sorted(best.tolist()) == list(range(args.n))
    drawn = score(args.model, matrix, cc.cc_init_tours(args.n, args.steps * args.batch, args.seed))
    print(f"{args.model}: learnt order {cost}, best of as many drawn orders {int(drawn.min())}, their mean {float(drawn.double().mean()):.0f}")


if __name__ == "__main__":
    main()
