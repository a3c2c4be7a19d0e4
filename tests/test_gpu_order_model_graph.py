"""The order model's calls in captured graphs, on other streams and after poisoned LDS: the same bits as eager calls."""
import pytest
import torch

import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


class Step:
    """A training step on buffers of its own: every call of the order model, forward and backward."""

    def __init__(self, b, t, v, d, dtype, placed):
        g = torch.Generator(device="cuda").manual_seed(7)
        self.b, self.t, self.v, self.d, self.placed = b, t, v, d, placed
        self.table = torch.randn(v + 1, d, generator=g, device="cuda").to(dtype)
        self.gates = torch.randn(b, t, d, generator=g, device="cuda").to(dtype)
        self.out = (torch.randn(d, v, generator=g, device="cuda") / d ** 0.5).to(dtype)
        self.tokens = torch.empty(b, t, dtype=torch.int32, device="cuda")
        self.old = torch.empty(b, t, device="cuda")
        self.advantage = torch.empty(b, device="cuda")
        self.lengths = torch.empty(b, dtype=torch.int32, device="cuda")
        self.h0 = torch.empty(b, d, device="cuda")
        self.fill(0)

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(100 + seed)
        self.tokens.copy_(torch.rand(self.b, self.v, generator=g, device="cuda").argsort(1)[:, :self.t])
        self.old.copy_(-2 + 0.1 * torch.randn(self.b, self.t, generator=g, device="cuda"))
        self.advantage.copy_(torch.randn(self.b, generator=g, device="cuda"))
        self.lengths.copy_(torch.randint(0, self.t + 1, (self.b,), generator=g, device="cuda"))
        self.h0.copy_(torch.randn(self.b, self.d, generator=g, device="cuda"))

    def run(self, stream=None):
        s = dict(stream=stream)
        x = cc.cc_embed(self.table, self.tokens, 2.0, **s)
        h, last, states = cc.cc_gated_scan(x, self.gates, self.h0, self.lengths, save_states=True, **s)
        logits = self.logits
        lp, rows = cc.cc_token_logprob(logits, self.tokens, None, self.placed, 0.5, **s)
        dlp = cc.cc_token_logprob_backward(logits, self.tokens, None, self.placed, 0.5, rows, lp, **s)
        p = cc.cc_policy_loss(logits, self.tokens, self.old, self.advantage, self.old, None, self.placed, 0.5, kl_coef=0.1, mean="orders", **s)
        q = cc.cc_preference_loss(logits, self.tokens, self.old, None, self.placed, 0.5, **s)
        gx, gg, g0 = cc.cc_gated_scan_backward(x, self.gates, states, h, last, self.lengths, **s)
        gt = cc.cc_embed_backward(gx, self.tokens, self.v + 1, 2.0, **s)
        return [x, h, last, lp, dlp, *p, *q, gx, gg, g0, gt]

    def prepare(self):
        self.logits = torch.randn(self.b, self.t, self.v, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(self.table.dtype)
        return self


CASES = [(6, 40, 50, 24, torch.float32, True), (4, 300, 700, 33, torch.bfloat16, True), (2, 3, 9000, 70, torch.float16, False),
         (2, 600, 1500, 16, torch.float32, False)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_graph_replays_equal_eager_calls(case):
    say(f"order model graph {case}")
    step = Step(*case).prepare()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step.run()
    for seed in range(4):
        step.fill(seed)
        want = [t.clone() for t in step.run()]
        torch.cuda.synchronize()
        for t in captured:
            if t.is_floating_point():
                t.fill_(77.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), seed


@pytest.mark.parametrize("case", CASES[:2], ids=str)
def test_another_stream(case):
    """Enqueued on a stream that is not the current one, with workspaces that the binding makes and drops."""
    step = Step(*case).prepare()
    want = [t.clone() for t in step.run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step.run(side)
    noise = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]      # takes freed blocks if they may be taken
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all((n == 3).all() for n in noise)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_lds_that_was_not_written_is_not_read(case, monkeypatch):
    step = Step(*case).prepare()
    want = [t.clone() for t in step.run()]
    monkeypatch.setenv("CC_LDS_POISON", "1")
    got = step.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_caller_s_workspaces():
    step = Step(*CASES[1]).prepare()
    want = [t.clone() for t in step.run()]
    b, t, v, d = step.b, step.t, step.v, step.d
    x, h, last = want[:3]
    ws = torch.full((max(cc.cc_token_workspace_bytes(b, t), cc.cc_embed_workspace_bytes(v + 1, d, b * t),
                         cc.cc_gated_scan_workspace_bytes(b, t, d)),), 0xA5, dtype=torch.uint8, device="cuda")
    p = cc.cc_policy_loss(step.logits, step.tokens, step.old, step.advantage, step.old, None, True, 0.5, kl_coef=0.1, mean="orders", workspace=ws)
    assert all(torch.equal(a, c) for a, c in zip(p, want[5:8]))
    q = cc.cc_preference_loss(step.logits, step.tokens, step.old, None, True, 0.5, workspace=ws)
    assert all(torch.equal(a, c) for a, c in zip(q, want[8:12]))
    gt = cc.cc_embed_backward(want[12], step.tokens, v + 1, 2.0, workspace=ws)
    assert torch.equal(gt, want[15])
    small = ws[:256]
    with pytest.raises(cc.CCError):
        cc.cc_embed_backward(want[12], step.tokens, v + 1, 2.0, workspace=small)
    with pytest.raises(cc.CCError):
        cc.cc_policy_loss(step.logits, step.tokens, step.old, step.advantage, workspace=small)
