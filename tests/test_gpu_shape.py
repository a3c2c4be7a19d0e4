"""Shaped logits and their gradient against the definition in 64 bits."""
import math

import pytest
import torch

import layers_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
DTYPES = [F32, F16, BF16]
# below a vector, odd, on both sides of every length that a wavefront's vectors hold, stretches
VOCABS = [1, 5, 8, 31, 64, 255, 257, 511, 513, 1000, 1025, 2047, 2048, 2049, 4096, 4101, 9000]


def inputs(b, t, v, length, dtype, seed=0, placed=False, ragged=True):
    g = torch.Generator().manual_seed(seed)
    logits = (3 * torch.randn(b, t, v, generator=g)).to(dtype)
    history = torch.randint(0, v, (b, length), generator=g, dtype=torch.int32)
    history[torch.rand(b, length, generator=g) < 0.1] = -1
    history[torch.rand(b, length, generator=g) < 0.05] = v
    if length > 4:
        history[:, 2] = -2 ** 31
        history[:, 3] = 2 ** 31 - 1
        history[:, 1] = history[:, 0]
    lengths = torch.randint(0, max(1, length - t // 2) + 1, (b,), generator=g, dtype=torch.int32)
    if ragged and b > 2:
        lengths[0], lengths[1], lengths[2] = 0, length + 9, -3
    starts = torch.randint(0, max(1, length // 2), (b,), generator=g, dtype=torch.int32)
    penalties = torch.stack([0.5 + torch.rand(b, generator=g), torch.randn(b, generator=g), torch.randn(b, generator=g)], 1)
    if placed:
        penalties[:, 0], penalties[:, 1], penalties[:, 2] = 1.0, math.inf, 0.0
    bias = torch.randn(b, v, generator=g)
    bias[:, ::5] = -math.inf
    allowed = torch.randint(-2 ** 31, 2 ** 31, (b, t, (v + 31) // 32), generator=g, dtype=torch.int64).to(torch.int32)
    allowed[-1, -1] = 0
    return logits, history, lengths, penalties, starts, bias, allowed


def check(args, seed=9):
    logits = args[0]
    dtype = logits.dtype
    dev = [a if a is None else a.cuda() for a in args]
    out = cc.cc_shape_logits(*dev)
    want, slope, size = ref.shaped(*args)
    gone = slope == 0
    got = out.cpu().double()
    assert (got[gone] == -math.inf).all()
    # a factor rounded and its product, the count's product and sums in 32 bits of what is at most `size`
    error = 6 * ref.U24 * size
    tol = ref.rounded(torch.where(gone, 0.0, want), dtype, error)
    assert ((got - want).abs() <= tol)[~gone].all(), float(((got - want).abs() - tol)[~gone].max())
    grad = torch.randn(logits.shape, generator=torch.Generator().manual_seed(seed)).to(dtype)
    grad[gone] = math.nan                                    # what a loss leaves where nothing is possible
    back = cc.cc_shape_logits_backward(grad.cuda(), *dev).cpu().double()
    want = torch.where(gone, 0.0, grad.double() * slope)
    assert ((back - want).abs() <= ref.rounded(want, dtype, 2 * ref.U24 * want.abs())).all()
    return out


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", VOCABS)
def test_single_positions(v, dtype):
    say(f"shape single {v} {dtype}")
    logits, history, lengths, penalties, starts, bias, allowed = inputs(6, 1, v, 50, dtype)
    check((logits, history, lengths, penalties, starts, bias, allowed))
    check((logits, history, lengths, penalties, None, None, None))
    check((logits, None, None, None, None, bias[0].contiguous(), None))
    check((logits, None, None, None, None, None, allowed))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", [7, 64, 250, 1000, 2100, 4100])
def test_sequences(v, dtype):
    say(f"shape sequences {v} {dtype}")
    for t, length in ((2, 1), (17, 30), (40, 20)):
        logits, history, lengths, penalties, starts, bias, allowed = inputs(4, t, v, length, dtype, t)
        check((logits, history, lengths, penalties, starts, bias, allowed))
        check((logits, history, None, penalties, None, bias[0].contiguous(), None))


@pytest.mark.parametrize("rows", [4096, 9000, 70000])
def test_rows_of_a_wavefront(rows):
    """So many rows that a wavefront takes several, one after the other: as single positions of the same history."""
    say(f"shape rows {rows}")
    t, v = 37, 20
    b = rows // t + 1
    logits, history, lengths, penalties, starts, _, _ = (a.cuda() for a in inputs(b, t, v, 45, BF16))
    got = cc.cc_shape_logits(logits, history, lengths, penalties, starts)
    for at in (0, 1, 15, 16, 17, 36):
        one = cc.cc_shape_logits(logits[:, at:at + 1].contiguous(), history, lengths + at, penalties, starts)
        assert torch.equal(got[:, at:at + 1], one)


@pytest.mark.parametrize("n", [8, 64, 300, 1000])
def test_placed_nodes_as_in_the_log_probability(n):
    """Orders as their own history: what is forbidden at a rank is what cc_token_logprob leaves out there."""
    say(f"shape placed {n}")
    g = torch.Generator(device="cuda").manual_seed(n)
    b = 3
    logits = torch.randn(b, n, n, generator=g, device="cuda")
    orders = torch.rand(b, n, generator=g, device="cuda").argsort(1).to(torch.int32)
    penalties = torch.tensor([1.0, math.inf, 0.0], device="cuda").repeat(b, 1)
    shaped = cc.cc_shape_logits(logits, orders, None, penalties)
    assert torch.equal(cc.cc_token_logprob(shaped, orders)[0], cc.cc_token_logprob(logits, orders, placed=True)[0])
    grad = torch.randn(b, n, generator=g, device="cuda")
    lp, rows = cc.cc_token_logprob(shaped, orders)
    through = cc.cc_shape_logits_backward(cc.cc_token_logprob_backward(shaped, orders, None, False, 1.0, rows, grad), logits, orders, None, penalties)
    lp, rows = cc.cc_token_logprob(logits, orders, placed=True)
    assert torch.equal(through, cc.cc_token_logprob_backward(logits, orders, None, True, 1.0, rows, grad))


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", [40, 2000, 5000])
def test_undefined_where_forbidden(v, dtype):
    say(f"shape undefined {v} {dtype}")
    logits, history, lengths, penalties, starts, bias, allowed = inputs(4, 3, v, 30, dtype, 3, placed=True)
    want, slope, _ = ref.shaped(logits, history, lengths, penalties, starts, bias, allowed)
    gone = slope == 0
    for bad in (math.nan, math.inf, -math.inf):
        z = logits.clone()
        z[gone] = bad
        dev = [a.cuda() for a in (z, history, lengths, penalties, starts, bias, allowed)]
        out = cc.cc_shape_logits(*dev).cpu()
        assert (out[gone] == -math.inf).all() and torch.isfinite(out[~gone]).all()
        back = cc.cc_shape_logits_backward(torch.ones_like(dev[0]), *dev).cpu()
        assert (back[gone] == 0).all() and torch.isfinite(back).all()
    z = logits.clone()
    z[~gone] = -math.inf
    assert (cc.cc_shape_logits(*(a.cuda() for a in (z, history, lengths, penalties, starts, bias, allowed))) == -math.inf).all()


def test_penalties_that_forbid_and_do_not():
    z = torch.tensor([[[1.0, -1.0, 2.0]]]).expand(5, 1, 3).contiguous().cuda()
    history = torch.tensor([[0, 1]], dtype=torch.int32).expand(5, 2).contiguous().cuda()
    lengths, starts = torch.full((5,), 2, dtype=torch.int32, device="cuda"), torch.full((5,), 1, dtype=torch.int32, device="cuda")
    inf = math.inf
    penalties = torch.tensor([[2.0, inf, 0.0], [2.0, 0.0, inf], [2.0, -inf, 0.0], [4.0, 0.0, 0.0], [1.0, 1.0, 1.0]], device="cuda")
    out = cc.cc_shape_logits(z, history, lengths, penalties, starts)[:, 0].tolist()
    assert out == [[0.5, -inf, 2.0], [0.5, -inf, 2.0], [0.5, inf, 2.0], [0.25, -4.0, 2.0], [1.0, -3.0, 2.0]]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", [33, 1000, 4500])
def test_strided_and_in_place(v, dtype):
    say(f"shape strided {v} {dtype}")
    b, t, length = 3, 5, 40
    args = [a.cuda() for a in inputs(b, t, v, length, dtype, 5)]
    logits, history, lengths, penalties, starts, bias, allowed = args
    want = cc.cc_shape_logits(*args)
    grad = torch.randn(b, t, v, device="cuda").to(dtype)
    want_back = cc.cc_shape_logits_backward(grad, *args)
    wide = torch.full((b, t + 1, v + 3), 7.0, device="cuda", dtype=dtype)
    wide[:, :t, 1:v + 1] = logits
    hist = torch.full((b, length + 3), 1, device="cuda", dtype=torch.int32)
    hist[:, 1:length + 1] = history
    bits = torch.full((t, b, allowed.shape[2] + 1), -1, device="cuda", dtype=torch.int32).transpose(0, 1)
    bits[:, :, :-1] = allowed
    biases = torch.zeros(b, v + 1, device="cuda")
    biases[:, 1:] = bias
    rest = (hist[:, 1:length + 1], lengths, penalties, starts, biases[:, 1:], bits[:, :, :-1])
    view = wide[:, :t, 1:v + 1]
    assert torch.equal(cc.cc_shape_logits(view, *rest), want)
    back = grad.clone()
    assert cc.cc_shape_logits_backward(back, view, *rest, grad_logits=back) is back and torch.equal(back, want_back)
    assert cc.cc_shape_logits(view, *rest, out=view) is view and torch.equal(view, want)
    assert (wide[:, t] == 7).all() and (wide[:, :, 0] == 7).all() and (wide[:, :, v + 1:] == 7).all()


def test_shared_masks_and_biases():
    b, t, v = 4, 6, 100
    logits, _, _, _, _, bias, allowed = (a.cuda() for a in inputs(b, t, v, 4, F32))
    one = allowed[:1, :1].expand(b, t, -1)
    assert torch.equal(cc.cc_shape_logits(logits, allowed=one), cc.cc_shape_logits(logits, allowed=one.contiguous()))
    assert torch.equal(cc.cc_shape_logits(logits, bias=bias[0].contiguous()), cc.cc_shape_logits(logits, bias=bias[:1].expand(b, v)))


def test_long_history():
    """More entries than a workgroup reads in a turn, one token in most of them."""
    say("shape long history")
    b, v, length = 3, 6000, 20011
    history = torch.full((b, length), 4097, dtype=torch.int32)
    history[:, ::3] = torch.randint(0, v, (b, len(range(0, length, 3))), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    logits = torch.randn(b, 1, v, generator=torch.Generator().manual_seed(2))
    check((logits, history, torch.tensor([length, length - 1, 5], dtype=torch.int32), torch.tensor([[1.5, 0.25, 0.001]] * b),
           torch.tensor([0, 10000, 0], dtype=torch.int32), None, None))
    check((logits[:, :, :1500].contiguous(), history % 1500, torch.tensor([length, length - 1, 5], dtype=torch.int32), torch.tensor([[1.5, 0.25, 0.001]] * b),
           None, None, None))


def test_nothing():
    assert cc.cc_shape_logits(torch.empty(0, 3, 5, device="cuda")).shape == (0, 3, 5)
    assert cc.cc_shape_logits(torch.empty(2, 0, 5, device="cuda")).shape == (2, 0, 5)
    z = torch.randn(2, 3, 5, device="cuda")
    assert torch.equal(cc.cc_shape_logits(z), z)
    empty = torch.empty(2, 0, dtype=torch.int32, device="cuda")
    assert torch.equal(cc.cc_shape_logits(z, empty, None, torch.ones(2, 3, device="cuda")), z)


def test_a_single_position_says_how_much_history_there_is():
    z, history = torch.randn(2, 1, 5, device="cuda"), torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="lengths"):
        cc.cc_shape_logits(z, history, None, torch.ones(2, 3, device="cuda"))


def repeated(z, r):
    """Logits whose tokens are all seen and do not count, with (r, 0, 0): the arguments behind them."""
    b, t, v = z.shape
    history = torch.arange(v, dtype=torch.int32, device="cuda").expand(b, v)
    lengths = torch.full((b,), v, dtype=torch.int32, device="cuda")
    return history, lengths, torch.tensor([r, 0.0, 0.0], device="cuda").repeat(b, 1), lengths + t


@pytest.mark.parametrize("v", [3, 40, 1000, 5000])
@pytest.mark.parametrize("r", [1.3, 0.7, 3.0, 1e10, 2.0 ** -130, 2.0 ** -140 * 3, 2.0 ** 127 * 1.7, 1e-30], ids=str)
def test_a_quotient_is_rounded_once(v, r):
    """z / r is off by a division's rounding and no more, whatever r is, and so is the gradient."""
    say(f"shape quotient {v} {r}")
    g = torch.Generator(device="cuda").manual_seed(v)
    r32 = float(torch.tensor(r))
    # quotients and products that a float holds
    size = min(1.0, r32 * 2.0 ** 120) * min(1e4, max(1.0, r32 * 2.0 ** -120))
    z = size * torch.randn(3, 2, v, generator=g, device="cuda")
    if r32 > 1e30:
        z = z.abs()
    rest = repeated(z, r)
    want = torch.where(z > 0, z.double() / r32, z.double() * r32)
    got = cc.cc_shape_logits(z, *rest)
    tol = 1.001 * ref.U24 * want.abs() + ref.BELOW[F32]
    assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() / want.abs()).max() / ref.U24)
    grad = size * torch.randn(3, 2, v, generator=g, device="cuda")
    want = torch.where(z > 0, grad.double() / r32, grad.double() * r32)
    held = want.abs() < torch.finfo(F32).max
    back = cc.cc_shape_logits_backward(grad, z, *rest)
    tol = 1.001 * ref.U24 * want.abs() + ref.BELOW[F32]
    assert ((back.double() - want).abs() <= tol)[held].all() and torch.isinf(back[~held]).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", [40, 3000])
def test_quotients_at_the_ends_of_the_range(v, dtype):
    """Infinities, undefined and the largest quotients, with divisors that have no reciprocal, or none of full length, too."""
    top = torch.finfo(dtype).max
    for r in (0.7, 2.0 ** -130, 2.0 ** -149, 2.0 ** 126 * 1.9, 1.5):
        r32 = float(torch.tensor(r))
        z = torch.zeros(2, 1, v, dtype=dtype)
        z[0, 0, :6] = torch.tensor([math.inf, -math.inf, math.nan, top, 1.0, 0.0]).to(dtype)
        edge = torch.tensor(min(top * r32, top), dtype=torch.float64).to(dtype)
        while float(edge) / r32 > top:
            edge = torch.nextafter(edge, torch.zeros((), dtype=dtype))
        z[0, 0, 6] = edge                                   # the largest with a quotient that the type holds
        z[1, 0, 0] = torch.finfo(dtype).tiny
        want = torch.where(z > 0, z.double() / r32, z.double() * r32).to(dtype)
        rest = repeated(z.cuda(), r)
        got = cc.cc_shape_logits(z.cuda(), *rest).cpu()
        back = cc.cc_shape_logits_backward(z.cuda(), z.cuda(), *rest).cpu()
        for out in (got, back):
            assert torch.equal(torch.isnan(out), torch.isnan(want)) and torch.equal(torch.isinf(out), torch.isinf(want))
            held = torch.isfinite(want)
            exact = torch.where(z > 0, z.double() / r32, z.double() * r32)[held]
            assert ((out[held].double() - exact).abs() <= ref.rounded(exact, dtype, 2 * ref.U24 * exact.abs())).all()
