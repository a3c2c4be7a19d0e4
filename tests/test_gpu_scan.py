"""The gated recurrence and its gradient against the definition in 64 bits."""
import pytest
import torch

import order_model_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say
from order_model_reference import DTYPES, finish, within

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


def make(b, t, d, dtype, seed=0, ragged=False, sharp=1.5):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(b, t, d, generator=g).to(dtype)
    gate = (sharp * torch.randn(b, t, d, generator=g) + 2).to(dtype)
    h0, gl = torch.randn(b, d, generator=g), torch.randn(b, d, generator=g)
    gh = torch.randn(b, t, d, generator=g).to(dtype)
    n = None
    if ragged:
        n = torch.randint(0, t + 1, (b,), generator=g, dtype=torch.int32)
        n[0] = 0
        n[-1] = t
        if b > 2:
            n[1] = t + 5                                    # more than there is: all of it
        if b > 3:
            n[2] = -3                                       # less than nothing: nothing
    return x, gate, h0, n, gh, gl


def check(b, t, d, name, ragged=False, seed=0, sharp=1.5, with_ends=True):
    say(f"scan b={b} t={t} d={d} {name} ragged={ragged}")
    dtype = DTYPES[name]
    x, gate, h0, n, gh, gl = make(b, t, d, dtype, seed, ragged, sharp)
    if not with_ends:
        h0 = gl = None
    dev = [v.cuda() if v is not None else None for v in (x, gate, h0, n, gh, gl)]
    h, last, states = cc.cc_gated_scan(*dev[:4], save_states=True)
    want, want_last, err, err_last = ref.scan(x, gate, h0, n)
    within(h, want, finish(want, err, dtype), "h")
    within(last, want_last, finish(want_last, err_last, torch.float32), "last")
    got = cc.cc_gated_scan_backward(dev[0], dev[1], states, dev[4], dev[5], dev[3])
    wants, errs = ref.scan_backward(x, gate, h0, n, gh, gl)
    for name_, g, w, e, kind in zip(("grad_x", "grad_gate", "grad_h0"), got, wants, errs, (dtype, dtype, torch.float32)):
        within(g, w, finish(w, e, kind), name_)
    again = cc.cc_gated_scan_backward(dev[0], dev[1], states, dev[4], dev[5], dev[3])
    assert all(torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,t,d", [(1, 1, 1), (3, 1, 7), (2, 15, 2), (2, 16, 33), (5, 17, 64), (1, 64, 128), (70, 31, 6), (4, 100, 250)])
def test_sizes(b, t, d, name):
    check(b, t, d, name)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("b,t,d", [(6, 1, 5), (7, 40, 9), (5, 300, 66)])
def test_ragged(b, t, d, name):
    check(b, t, d, name, ragged=True)


@pytest.mark.parametrize("b,t,d,ragged", [(1, 128, 4, False), (1, 1000, 3, False), (4, 513, 32, True), (2, 4099, 16, True), (1, 5000, 1, False)])
def test_long_and_split(b, t, d, ragged):
    check(b, t, d, "f32", ragged)
    check(b, t, d, "bf16", ragged)


def test_without_first_state_and_without_last_gradient():
    check(3, 50, 20, "f32", with_ends=False)
    check(2, 700, 5, "bf16", ragged=True, with_ends=False)


def test_gates_at_the_ends_of_their_range():
    """Gates that open and close entirely, and infinite ones: keep is 1 or 0, the other exactly 0 or 1."""
    check(2, 60, 10, "f32", sharp=60.0)
    x = torch.randn(1, 40, 4, generator=torch.Generator().manual_seed(4))
    gate = torch.full((1, 40, 4), float("inf"))
    gate[:, 10] = float("-inf")
    h, last, _ = cc.cc_gated_scan(x.cuda(), gate.cuda(), torch.full((1, 4), 3.0, device="cuda"))
    assert (h[:, :10] == 3).all() and torch.equal(h[:, 10:].cpu(), x[:, 10:11].expand(1, 30, 4)) and torch.equal(last.cpu(), x[:, 10])


def test_what_lies_beyond_a_length_is_not_read():
    x, gate, h0, _, gh, gl = make(3, 200, 10, torch.float32)
    n = torch.tensor([0, 77, 200], dtype=torch.int32)
    dirty = [v.clone() for v in (x, gate, gh)]
    for v in dirty:
        for i in range(3):
            v[i, int(n[i]):] = float("nan")
    def run(x, gate, gh):
        h, last, states = cc.cc_gated_scan(x.cuda(), gate.cuda(), h0.cuda(), n.cuda(), save_states=True)
        return (h, last, *cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, gh.cuda(), gl.cuda(), n.cuda()))
    for a, b in zip(run(x, gate, gh), run(*dirty)):
        assert torch.equal(a, b)


def test_no_positions_hand_the_state_through():
    h0 = torch.randn(3, 6, device="cuda")
    empty = torch.zeros(3, 0, 6, device="cuda")
    h, last, states = cc.cc_gated_scan(empty, empty, h0, save_states=True)
    assert h.shape == (3, 0, 6) and torch.equal(last, h0)
    gx, gg, g0 = cc.cc_gated_scan_backward(empty, empty, states, empty, h0)
    assert gx.shape == (3, 0, 6) and torch.equal(g0, h0)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 7])
def test_steps_make_the_scan(name, d):
    """T single steps with the state updated in place, as sampling does them, give what the scan gives, bit for bit."""
    x, gate, h0, _, _, _ = make(5, 30, d, DTYPES[name])
    x, gate, state = x.cuda(), gate.cuda(), h0.cuda().clone()
    h, last, _ = cc.cc_gated_scan(x, gate, h0.cuda())
    for t in range(30):
        step, same, _ = cc.cc_gated_scan(x[:, t:t + 1], gate[:, t:t + 1], state, last=state)
        assert same is state and torch.equal(step[:, 0], h[:, t])
    assert torch.equal(state, last)


@pytest.mark.parametrize("d", [16, 9])
def test_strides_and_odd_addresses(d):
    b, t = 3, 45
    for dtype in (torch.float32, torch.float16):
        x, gate, h0, n, gh, gl = make(b, t, d, dtype, 2, ragged=True)
        room = torch.full((b * t * (2 * d + 3) + 1,), 4.0, dtype=dtype, device="cuda")
        both = room[1:].view(t, b, 2 * d + 3).transpose(0, 1)          # time outermost, both halves in one row
        both[..., :d], both[..., d + 1:2 * d + 1] = x.cuda(), gate.cuda()
        xs, gs = both[..., :d], both[..., d + 1:2 * d + 1]
        out = torch.empty(b, t + 2, d + 1, dtype=dtype, device="cuda")
        out.fill_(8.0)
        h, last, states = cc.cc_gated_scan(xs, gs, h0.cuda(), n.cuda(), save_states=True, out=out[:, 1:t + 1, 1:])
        plain = cc.cc_gated_scan(x.cuda(), gate.cuda(), h0.cuda(), n.cuda(), save_states=True)
        assert torch.equal(h, plain[0]) and torch.equal(last, plain[1]) and torch.equal(states, plain[2])
        assert (out[:, 0] == 8).all() and (out[:, -1] == 8).all() and (out[..., 0] == 8).all()
        grads = torch.full_like(room, 6.0)
        into = grads[1:].view(t, b, 2 * d + 3).transpose(0, 1)
        got = cc.cc_gated_scan_backward(xs, gs, states, gh.cuda(), gl.cuda(), n.cuda(), grad_x=into[..., :d], grad_gate=into[..., d + 1:2 * d + 1])
        want = cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, gh.cuda(), gl.cuda(), n.cuda())
        assert all(torch.equal(p, q) for p, q in zip(got, want))
        assert (into[..., d] == 6).all() and (into[..., 2 * d + 1:] == 6).all()


def test_one_gradient_for_all_positions():
    """A broadcast gradient: strides of zero where it is read."""
    x, gate, h0, _, _, gl = make(3, 60, 8, torch.float32)
    h, last, states = cc.cc_gated_scan(x.cuda(), gate.cuda(), h0.cuda(), save_states=True)
    one = torch.randn(1, 1, 8, device="cuda").expand(3, 60, 8)
    got = cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, one, gl.cuda())
    want = cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, one.contiguous(), gl.cuda())
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_offsets_beyond_32_bits():
    b, t, d = 2, 3, 16
    apart = (1 << 31) + 64
    room = torch.empty(apart + t * d, dtype=torch.bfloat16, device="cuda")
    x, gate, h0, _, gh, gl = make(b, t, d, torch.bfloat16)
    far = torch.as_strided(room, (b, t, d), (apart, d, 1))
    far.copy_(x.cuda())
    say("scan: sequences 4.3 GB apart")
    h, last, states = cc.cc_gated_scan(far, gate.cuda(), h0.cuda(), save_states=True)
    want = cc.cc_gated_scan(x.cuda(), gate.cuda(), h0.cuda(), save_states=True)
    assert torch.equal(h, want[0]) and torch.equal(last, want[1])
    into = torch.as_strided(torch.empty_like(room), (b, t, d), (apart, d, 1))
    got = cc.cc_gated_scan_backward(far, gate.cuda(), states, gh.cuda(), gl.cuda(), grad_x=into)
    want = cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, gh.cuda(), gl.cuda())
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_gradient_against_differences():
    """The kernels' own loss in a direction: two losses in 32 bits differ by 2 eps <gradient, direction>.  h is exact to within
    the bound of the reference, and so is each loss to within sum(|weight| bound); the step is chosen so that this and the
    third derivative (of order one here, times eps^2) are small beside the slope."""
    b, t, d, eps = 2, 90, 6, 2.0 ** -6
    x, gate, h0, _, gh, gl = make(b, t, d, torch.float32, 11)
    g = torch.Generator().manual_seed(12)
    direction = [torch.randn(v.shape, generator=g) for v in (x, gate, h0)]
    h, last, states = cc.cc_gated_scan(x.cuda(), gate.cuda(), h0.cuda(), save_states=True)
    grads = cc.cc_gated_scan_backward(x.cuda(), gate.cuda(), states, gh.cuda(), gl.cuda())
    slope = sum(float((p.cpu().double() * q.double()).sum()) for p, q in zip(grads, direction))

    def loss(s):
        args = [(v + s * eps * q).cuda() for v, q in zip((x, gate, h0), direction)]
        h, last, _ = cc.cc_gated_scan(*args)
        return float((h.double().cpu() * gh.double()).sum() + (last.double().cpu() * gl.double()).sum())

    # Richardson: the term in eps^2 is taken out by a second pair of losses at twice the step
    near, far = (loss(1) - loss(-1)) / (2 * eps), (loss(2) - loss(-2)) / (4 * eps)
    estimate = (4 * near - far) / 3
    _, _, err, err_last = ref.scan(x, gate, h0, None)
    noise = float((err * gh.abs()).sum() + (err_last * gl.abs()).sum()) * 2 / eps
    assert abs(estimate - slope) <= noise + 2e-4 * abs(far - near) + 1e-3 * abs(slope)


def test_states_beyond_32_bits_without_positions():
    """2^30 channels and no position: the states lie beyond 4 GB where the tensors of 16 bits do not."""
    b, d = (1 << 30) // 1000 + 7, 1000
    say("scan: 4.3 GB of states, no positions")
    h0 = torch.arange(b * d, dtype=torch.int32, device="cuda").view(torch.float32).view(b, d)
    empty = torch.empty(b, 0, d, dtype=torch.bfloat16, device="cuda")
    _, last, states = cc.cc_gated_scan(empty, empty, h0, save_states=True)
    assert torch.equal(last.view(torch.int32), h0.view(torch.int32))
    last.zero_()
    _, _, g0 = cc.cc_gated_scan_backward(empty, empty, states, empty, h0, grad_h0=last)
    assert torch.equal(g0.view(torch.int32), h0.view(torch.int32))
