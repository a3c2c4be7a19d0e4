"""Gates about the size from which on the recurrence takes them apart: whatever lies in the same chunk, a position gives the
same bits as alone."""
import pytest
import torch

import order_model_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say
from order_model_reference import DTYPES, finish, within
from test_gpu_scan import make

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


def steep(b, t, d, dtype, some):
    """Gates of some units, and in the chunks of every other 16 positions a few about +-64 and beyond."""
    x, gate, h0, n, gh, gl = make(b, t, d, dtype, seed=t + d)
    g = torch.Generator().manual_seed(d)
    far = torch.tensor([63.75, 64.0, 64.5, -63.75, -64.0, -64.5, 90.0, -100.0, 3e4, -3e4])
    pick = far[torch.randint(0, len(far), gate.shape, generator=g)].to(dtype)
    where = torch.rand(gate.shape, generator=g) < some
    where[:, (torch.arange(t) // 16) % 2 == 1] = False
    return x, torch.where(where, pick, gate), h0, n, gh, gl


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("b,t,d", [(3, 70, 8), (2, 40, 7), (1, 33, 1), (5, 64, 130)])
def test_gates_of_all_sizes_in_one_chunk(b, t, d, name):
    say(f"scan of steep gates b={b} t={t} d={d} {name}")
    dtype = DTYPES[name]
    x, gate, h0, n, gh, gl = steep(b, t, d, dtype, 0.05)
    dev = [v.cuda() for v in (x, gate, h0)]
    h, last, states = cc.cc_gated_scan(*dev, save_states=True)
    want, want_last, err, err_last = ref.scan(x, gate, h0, None)
    within(h, want, finish(want, err, dtype), "h")
    within(last, want_last, finish(want_last, err_last, torch.float32), "last")
    got = cc.cc_gated_scan_backward(dev[0], dev[1], states, gh.cuda(), gl.cuda())
    wants, errs = ref.scan_backward(x, gate, h0, None, gh, gl)
    for what, g, w, e, kind in zip(("grad_x", "grad_gate", "grad_h0"), got, wants, errs, (dtype, dtype, torch.float32)):
        within(g, w, finish(w, e, kind), what)
    state = dev[2].clone()
    for i in range(t):
        step, _, _ = cc.cc_gated_scan(dev[0][:, i:i + 1], dev[1][:, i:i + 1], state, last=state)
        assert torch.equal(step[:, 0], h[:, i])
    assert torch.equal(state, last)


@pytest.mark.parametrize("d", [8, 9])
def test_a_neighbours_gates_do_not_show(d):
    """Channels whose gates are mild have the same bits whether another channel's are or not."""
    x, gate, h0, n, gh, gl = make(2, 64, d, torch.bfloat16, seed=5)
    other = gate.clone()
    other[:, ::3, 0] = 80.0
    dev = [v.cuda() for v in (x, h0, gh, gl)]
    results = []
    for g in (gate, other):
        h, last, states = cc.cc_gated_scan(dev[0], g.cuda(), dev[1], save_states=True)
        results.append([h, last, *cc.cc_gated_scan_backward(dev[0], g.cuda(), states, dev[2], dev[3])])
    for one, two in zip(*results):
        assert torch.equal(one[..., 1:], two[..., 1:])
