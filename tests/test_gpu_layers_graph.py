"""A policy's step with norm, products in 8 bits and shaped logits: together as a sampling step and its training use them, in captured graphs,
on other streams and after poisoned LDS: the same bits as eager calls."""
import math

import pytest
import torch

import layers_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


class Step:
    """Two layers of a recurrence with a norm between them, an 8-bit head, shaped logits and their log-probability; the same
    head in the type and its gradients down to the first layer's output."""

    def __init__(self, b, t, v, d, dtype, placed):
        g = torch.Generator(device="cuda").manual_seed(7)

        def randn(*shape):
            return torch.randn(*shape, generator=g, device="cuda")

        self.b, self.t, self.v, self.d, self.placed = b, t, v, d, placed
        self.table, self.gates = randn(v + 1, d).to(dtype), randn(b, t, d).to(dtype)
        self.weight = 1 + 0.1 * randn(d)
        self.head = (randn(v, d) / d ** 0.5).to(dtype)
        self.bias = randn(v)
        self.tokens = torch.empty(b, t, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(b, dtype=torch.int32, device="cuda")
        self.grad = torch.empty(b, t, device="cuda")
        penalty = [1.0, math.inf, 0.0] if placed else [1.3, 0.5, 0.25]
        self.penalties = torch.tensor(penalty, device="cuda").repeat(b, 1)
        self.allowed = torch.randint(-2 ** 31, 2 ** 31, (b, t, (v + 31) // 32), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        self.fill(0)

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(100 + seed)
        self.tokens.copy_(torch.rand(self.b, self.v, generator=g, device="cuda").argsort(1)[:, :self.t])
        self.grad.copy_(torch.randn(self.b, self.t, generator=g, device="cuda"))
        if not self.placed:
            self.lengths.copy_(torch.randint(0, 3, (self.b,), generator=g, device="cuda"))

    def shape(self):
        return dict(history=self.tokens, lengths=self.lengths, penalties=self.penalties, bias=self.bias, allowed=None if self.placed else self.allowed)

    def run(self, stream=None):
        s = dict(stream=stream)
        x = cc.cc_embed(self.table, self.tokens, 2.0, **s)
        h, _, states = cc.cc_gated_scan(x, self.gates, save_states=True, **s)
        res = cc.cc_rms_norm(h, self.weight, x, quantized=True, save_rstd=True, **s)
        w, w_scale = cc.cc_quantize_rows(self.head, **s)
        logits = cc.cc_product_i8(res.q, res.scale, w, w_scale, self.bias, **s)
        shaped = cc.cc_shape_logits(logits, **self.shape(), **s)
        lp, rows = cc.cc_token_logprob(shaped, self.tokens, **s)
        dshaped = cc.cc_token_logprob_backward(shaped, self.tokens, None, False, 1.0, rows, self.grad, **s)
        dlogits = cc.cc_shape_logits_backward(dshaped, logits, **self.shape(), **s)
        gh, gw = cc.cc_rms_norm_backward(res.out, res.sum, res.rstd, self.weight, x, **s)
        gx, gg, _ = cc.cc_gated_scan_backward(x, self.gates, states, gh, **s)
        return [x, h, res.out, res.sum, res.q, res.scale, res.rstd, w, w_scale, logits, shaped, lp, dshaped, dlogits, gh, gw, gx, gg]


CASES = [(6, 40, 50, 24, torch.float32, True), (4, 300, 700, 136, torch.bfloat16, True), (2, 3, 9000, 272, torch.float16, False),
         (2, 200, 4100, 1024, torch.bfloat16, False)]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_graph_replays_equal_eager_calls(case):
    say(f"layers graph {case}")
    step = Step(*case)
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
            t.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(captured, want)), seed


@pytest.mark.parametrize("case", CASES, ids=str)
def test_another_stream(case):
    say(f"layers stream {case}")
    step = Step(*case)
    want = [t.clone() for t in step.run()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step.run(side)
    noise = [torch.full((1 << 20,), 3.0, device="cuda") for _ in range(8)]      # takes freed blocks if they may be taken
    side.synchronize()
    assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(got, want))
    assert all((n == 3).all() for n in noise)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_lds_that_was_not_written_is_not_read(case, monkeypatch):
    say(f"layers poison {case}")
    step = Step(*case)
    want = [t.clone() for t in step.run()]
    monkeypatch.setenv("CC_LDS_POISON", "1")
    got = step.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(got, want))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_the_step_in_64_bits(case):
    """The 8-bit head's logits, from what the calls before it gave, and each row's log-probability among what is left."""
    say(f"layers step {case}")
    step = Step(*case)
    x, h, out, total, q, scale, rstd, w, w_scale, logits, shaped, lp = step.run()[:12]
    want = ref.product(q.view(-1, step.d), scale.view(-1), w, w_scale, step.bias).view_as(logits)
    assert ((logits.double() - want).abs() <= 4 * ref.U24 * (want - step.bias.double()).abs() + 2 * ref.U24 * want.abs()).all()
    # an int8 row is off by half a step of its scale an element
    exact = out.double() - q.double() * scale.double().unsqueeze(-1)
    assert (exact.abs() <= ref.rounded(out.double(), out.dtype, 0.5001 * scale.double().unsqueeze(-1) + 4 * ref.U24 * out.double().abs())).all()
    z = shaped.double()
    chosen = z.gather(2, step.tokens.long().unsqueeze(2)).squeeze(2)
    want = chosen - torch.logsumexp(z, 2)
    both = torch.isneginf(chosen)
    assert (lp[both] == -math.inf).all() and ((lp.double() - want).abs()[~both] <= 1e-5).all()


def test_workspaces_of_the_caller():
    step = Step(*CASES[1])
    n, d = step.b * step.t, step.d
    res = step.run()
    out, total, rstd, x, gh, gw = res[2], res[3], res[6], res[0], res[14], res[15]
    ws = torch.full((cc.cc_rms_norm_workspace_bytes(n, d),), 0xA5, dtype=torch.uint8, device="cuda")
    got = cc.cc_rms_norm_backward(out, total, rstd, step.weight, x, workspace=ws)
    assert torch.equal(got[0], gh) and torch.equal(got[1], gw)
    with pytest.raises(cc.CCError):
        cc.cc_rms_norm_backward(out, total, rstd, step.weight, x, workspace=ws[:-256])
    q, scale, w, w_scale, logits = res[4], res[5], res[7], res[8], res[9]
    for m in (n, 40):
        qm, sm = q.view(-1, d)[:m], scale.view(-1)[:m]
        ws = torch.full((max(256, cc.cc_product_i8_workspace_bytes(m, step.v, d)),), 0xA5, dtype=torch.uint8, device="cuda")
        assert torch.equal(cc.cc_product_i8(qm, sm, w, w_scale, step.bias, workspace=ws), logits.view(-1, step.v)[:m])
