"""Ratios and divergences that 32 bits do not hold: a position without an advantage, or a divergence whose coefficient is zero, has
no part in loss and gradient even so."""
import pytest
import torch

import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


@pytest.mark.parametrize("v", [12, 2500])
@pytest.mark.parametrize("old", [-200.0, float("-inf")])
def test_no_advantage_and_a_ratio_beyond_the_range(v, old):
    say(f"policy loss v={v} old={old}")
    logits = torch.randn(3, 5, v, generator=torch.Generator().manual_seed(v)).cuda()
    tokens = torch.arange(5, dtype=torch.int32).expand(3, 5).contiguous().cuda()
    lp, _ = cc.cc_token_logprob(logits, tokens)
    res = cc.cc_policy_loss(logits, tokens, torch.full((3, 5), old, device="cuda"), torch.zeros(3, device="cuda"), lp, kl_coef=0.0)
    assert torch.equal(res.logprob, lp) and float(res.stats[0]) == 0 and float(res.stats[2]) == 0
    assert (res.grad_logits == 0).all()
    # an advantage above zero is held at the border: its gain is 1.2 times the advantage, and nothing pulls
    res = cc.cc_policy_loss(logits, tokens, torch.full((3, 5), old, device="cuda"), torch.full((3,), 0.5, device="cuda"), clip_high=0.2)
    # 0.6 with the roundings of the border, of its product and of 15 weights and terms, in 32 bits each
    assert abs(float(res.stats[0]) + 0.6) <= 0.6 * 20 * 2.0 ** -24 and (res.grad_logits == 0).all()


@pytest.mark.parametrize("v", [12, 2500])
def test_a_divergence_beyond_the_range_that_counts_for_nothing(v):
    say(f"policy loss v={v}")
    logits = torch.randn(2, 4, v, generator=torch.Generator().manual_seed(v)).cuda()
    tokens = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    lp, _ = cc.cc_token_logprob(logits, tokens)
    advantage = torch.tensor([1.0, -1.0], device="cuda")
    far = cc.cc_policy_loss(logits, tokens, lp, advantage, torch.full((2, 4), 300.0, device="cuda"), kl_coef=0.0)
    none = cc.cc_policy_loss(logits, tokens, lp, advantage)
    assert torch.equal(far.grad_logits, none.grad_logits) and float(far.stats[0]) == float(none.stats[0])
