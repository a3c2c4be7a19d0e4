"""Log-probabilities, policy loss and preference loss against their definitions in 64 bits."""
import pytest
import torch

import order_model_reference as ref
import paper_2105_14088_amd as cc
from gpu_util import say
from order_model_reference import DTYPES, U, finish, within

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]

SCALE = 0.75


def make(b, t, v, dtype, seed=0, placed=False, masked=True):
    g = torch.Generator().manual_seed(seed)
    logits = (2 * torch.randn(b, t, v, generator=g)).to(dtype)
    if placed:
        tokens = torch.rand(b, v, generator=g).argsort(1)[:, :t].to(torch.int32)
    else:
        tokens = torch.randint(0, v, (b, t), generator=g, dtype=torch.int32)
    mask = None
    if masked:
        mask = torch.rand(b, t, generator=g) < 0.8
        mask[0] = False
        mask[-1] = True
    return logits, tokens.contiguous(), mask


def dev(*ts):
    return [None if x is None else x.cuda() for x in ts]


def check_logprob(logits, tokens, mask, placed, seed=1):
    dtype = logits.dtype
    p, rest, lp, valid, rel = ref.rows(logits, tokens, mask, placed, SCALE)
    z, k, m = dev(logits, tokens, mask)
    got, rows = cc.cc_token_logprob(z, k, m, placed, SCALE)
    within(got, lp, finish(lp, lp.abs() * U + rel, torch.float32), "logprob")
    slope = torch.randn(lp.shape, generator=torch.Generator().manual_seed(seed))
    want = ref.grad_logits(p, rest, tokens, valid, slope.double() * SCALE * 4)
    grad = cc.cc_token_logprob_backward(z, k, m, placed, SCALE, rows, slope.cuda(), grad_scale=4.0)
    within(grad, want, finish(want, want.abs() * (2 * rel + 8 * U), dtype), "gradient")
    place = z.clone()
    cc.cc_token_logprob_backward(place, k, m, placed, SCALE, rows, slope.cuda(), grad_scale=4.0, grad_logits=place)
    assert torch.equal(place, grad)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [1, 2, 7, 8, 9, 31, 33, 64, 65, 100, 129, 255, 257, 500, 513, 1000, 1024])
def test_orders(v, name):
    t = min(v, 40)
    say(f"logprob placed v={v} t={t} {name}")
    check_logprob(*make(3, t, v, DTYPES[name], v, placed=True), True)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,t,v", [(1, 1, 1), (2, 3, 5), (300, 1, 12), (5, 7, 1023), (2, 3, 1025), (2, 2, 2048), (2, 3, 4099), (1, 3, 16385),
                                   (2, 2, 50001), (1, 2, 65536), (1, 2, 131079), (1, 1, 300007)])
def test_any_vocabulary(b, t, v, name):
    say(f"logprob b={b} t={t} v={v} {name}")
    check_logprob(*make(b, t, v, DTYPES[name], v, masked=b > 1), False)


@pytest.mark.parametrize("b,t,v", [(1, 64, 64), (40, 8, 8), (200, 3, 100), (2, 130, 300), (9, 1, 1024)])
def test_whole_orders_and_short_ones(b, t, v):
    check_logprob(*make(b, t, v, torch.float32, 5, placed=True, masked=b > 1), True)


def test_tokens_that_are_none():
    """Out of range tokens do not count; a node that stands twice is left out after its first place only for others."""
    logits, tokens, _ = make(3, 12, 20, torch.float32, 3, placed=True, masked=False)
    tokens[0, 3], tokens[0, 4], tokens[1, 0], tokens[2, 7] = -1, 20, 2 ** 31 - 1, -(2 ** 31)
    tokens[2, 5] = tokens[2, 1]
    for placed in (False, True):
        check_logprob(logits, tokens, None, placed)


def test_what_is_left_out_has_no_effect():
    """NaN and infinities at nodes that are placed and in positions that do not count change nothing."""
    logits, tokens, mask = make(4, 30, 30, torch.float32, 6, placed=True)
    dirty = logits.clone()
    for b in range(4):
        for t in range(30):
            for at, j in enumerate(tokens[b, :t].tolist()):
                dirty[b, t, j] = (float("nan"), float("inf"), float("-inf"))[at % 3]
            if not mask[b, t]:
                dirty[b, t] = float("nan")
    slope = torch.randn(4, 30).cuda()
    outs = []
    for z in (logits, dirty):
        lp, rows = cc.cc_token_logprob(z.cuda(), tokens.cuda(), mask.cuda(), True, SCALE)
        outs.append((lp, cc.cc_token_logprob_backward(z.cuda(), tokens.cuda(), mask.cuda(), True, SCALE, rows, slope)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert torch.isfinite(outs[1][1]).all()


@pytest.mark.parametrize("v", [6, 300, 5000])
def test_logits_of_minus_infinity_and_of_the_lowest_value(v):
    logits, tokens, _ = make(2, 4, v, torch.float32, 8, masked=False)
    logits[0, 0, 1:] = float("-inf")
    tokens[0, 0] = 0                                            # the only candidate: certain
    logits[0, 1] = float("-inf")                                # none at all
    logits[0, 2, :3] = float("-inf")
    tokens[0, 2] = 1                                            # impossible
    logits[0, 3] = torch.finfo(torch.float32).min / 2
    logits[1, 0, : v // 2] = torch.finfo(torch.float32).min
    tokens[1, 0] = v - 1
    check_logprob(logits, tokens, None, False)
    lp, _ = cc.cc_token_logprob(logits.cuda(), tokens.cuda(), None, False, SCALE)
    assert float(lp[0, 0]) == 0 and float(lp[0, 1]) == float("-inf") and float(lp[0, 2]) == float("-inf")


def test_a_nan_stays_in_its_row():
    logits, tokens, _ = make(2, 3, 2000, torch.float32, 8, masked=False)
    clean, _ = cc.cc_token_logprob(logits.cuda(), tokens.cuda(), None, False, SCALE)
    logits[1, 1, 77] = float("nan")
    lp, _ = cc.cc_token_logprob(logits.cuda(), tokens.cuda(), None, False, SCALE)
    assert torch.isnan(lp[1, 1]) and int(torch.isnan(lp).sum()) == 1
    keep = ~torch.isnan(lp)
    assert torch.equal(lp[keep], clean[keep])


def test_strides_and_odd_addresses():
    for b, t, v in ((3, 9, 33), (2, 3, 1501)):
        for dtype in (torch.float32, torch.bfloat16):
            logits, tokens, mask = make(b, t, v, dtype, 9)
            room = torch.full((t * b * (v + 2) + 1,), 3.0, dtype=dtype, device="cuda")
            odd = room[1:].view(t, b, v + 2).transpose(0, 1)[..., 1:v + 1]
            odd.copy_(logits.cuda())
            k, m = dev(tokens, mask)
            lp, rows = cc.cc_token_logprob(odd, k, m, False, SCALE)
            want, want_rows = cc.cc_token_logprob(logits.cuda(), k, m, False, SCALE)
            assert torch.equal(lp, want) and torch.equal(rows, want_rows)
            slope = torch.randn(b, t, device="cuda")
            grads = torch.full_like(room, 3.0)
            into = grads[1:].view(t, b, v + 2).transpose(0, 1)[..., 1:v + 1]
            cc.cc_token_logprob_backward(odd, k, m, False, SCALE, rows, slope, grad_logits=into)
            assert torch.equal(into, cc.cc_token_logprob_backward(logits.cuda(), k, m, False, SCALE, rows, slope))
            assert (grads[1:].view(t, b, v + 2)[..., 0] == 3).all() and (grads[1:].view(t, b, v + 2)[..., -1] == 3).all()


def test_one_row_of_logits_for_all_orders():
    """A policy that does not look at the order's past: logits with a stride of zero over orders."""
    logits, tokens, mask = make(6, 10, 10, torch.float32, 4, placed=True)
    shared = logits[:1].cuda().expand(6, 10, 10)
    k, m = dev(tokens, mask)
    lp, rows = cc.cc_token_logprob(shared, k, m, True, SCALE)
    assert torch.equal(lp, cc.cc_token_logprob(shared.contiguous(), k, m, True, SCALE)[0])


def test_offsets_beyond_32_bits():
    b, t, v = 2, 2, 1500
    apart = (1 << 31) + 64
    room = torch.empty(apart + t * v, dtype=torch.bfloat16, device="cuda")
    logits, tokens, _ = make(b, t, v, torch.bfloat16, 2)
    far = torch.as_strided(room, (b, t, v), (apart, v, 1))
    far.copy_(logits.cuda())
    say("token: orders 4.3 GB apart")
    for cut in (v, 900):
        z, k = far[..., :cut], tokens.clamp(max=cut - 1).cuda()
        near = z.contiguous()
        lp, rows = cc.cc_token_logprob(z, k, None, False, SCALE)
        want, rows2 = cc.cc_token_logprob(near, k, None, False, SCALE)
        assert torch.equal(lp, want)
        slope = torch.randn(b, t, device="cuda")
        want = cc.cc_token_logprob_backward(near, k, None, False, SCALE, rows2, slope)
        kept = near.clone()
        cc.cc_token_logprob_backward(z, k, None, False, SCALE, rows, slope, grad_logits=z)
        assert torch.equal(z, want)
        z.copy_(kept)


# ---------------------------------------------------------------------------------------------------------- policy


def policy_inputs(lp, per_token, seed=0):
    """Old log-probabilities whose ratios stay clear of the clip's borders (0.8, 1.25): the slope jumps there."""
    g = torch.Generator().manual_seed(seed)
    ratio = torch.tensor([0.5, 0.7, 0.9, 1.0, 1.1, 1.2, 1.4, 2.0], dtype=torch.float64)
    ratio = ratio[torch.randint(0, 8, lp.shape, generator=g)]
    old = torch.where(torch.isfinite(lp), lp, 0.0) - torch.log(ratio)
    other = torch.where(torch.isfinite(lp), lp, 0.0) + 0.3 * torch.randn(lp.shape, generator=g)
    adv = torch.randn(lp.shape if per_token else lp.shape[:1], generator=g)
    return old.float(), other.float(), adv


def check_policy(logits, tokens, mask, placed, mean, per_token=False, with_ref=True, coef=0.1):
    dtype = logits.dtype
    b, t, v = logits.shape
    p, rest, lp, valid, rel = ref.rows(logits, tokens, mask, placed, SCALE)
    old, other, adv = policy_inputs(lp, per_token)
    if not with_ref:
        other = None
    stats, slope, moved, total = ref.policy(lp, valid, old, other, adv, 0.2, 0.25, coef, mean)
    scale = 128.0 if dtype is torch.float16 else 1.0
    z, k, m, o, r, a = dev(logits, tokens, mask, old, other, adv)
    res = cc.cc_policy_loss(z, k, o, a, r, m, placed, SCALE, 0.2, 0.25, coef, mean, grad_scale=scale)
    lp_err = lp.abs() * U + rel
    within(res.logprob, lp, finish(lp, lp_err, torch.float32), "logprob")
    # an exponential of a difference: the difference's error, its rounding, the function's last bits; weights and products
    slope_err = moved * (rel + 16 * U)
    loss_err = float(total) * (rel + 16 * U)
    want_stats_err = torch.tensor([loss_err, loss_err / max(coef, 1e-3) + 16 * U * float(stats[1]), 16 * U * float(stats[2])], dtype=torch.float64)
    within(res.stats, stats, finish(stats, want_stats_err, torch.float32) + stats.abs() * U, "stats")
    want = ref.grad_logits(p, rest, tokens, valid, slope * SCALE * scale)
    err = ref.grad_logits(p, -rest, tokens, valid, slope_err * SCALE * scale).abs() + want.abs() * (2 * rel + 8 * U)
    within(res.grad_logits, want, finish(want, err, dtype), "gradient")
    again = cc.cc_policy_loss(z, k, o, a, r, m, placed, SCALE, 0.2, 0.25, coef, mean, grad_scale=scale)
    assert all(torch.equal(x, y) for x, y in zip(res, again))
    bare = cc.cc_policy_loss(z, k, o, a, r, m, placed, SCALE, 0.2, 0.25, coef, mean, grad=False)
    assert bare.grad_logits is None and torch.equal(bare.stats, res.stats) and torch.equal(bare.logprob, res.logprob)
    place = z.clone()
    cc.cc_policy_loss(place, k, o, a, r, m, placed, SCALE, 0.2, 0.25, coef, mean, grad_scale=scale, grad_logits=place)
    assert torch.equal(place, res.grad_logits)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("mean", ["tokens", "orders"])
@pytest.mark.parametrize("b,t,v,placed", [(1, 1, 1, False), (3, 8, 8, True), (50, 5, 9, True), (5, 64, 64, True), (2, 33, 500, True),
                                          (4, 6, 1000, False), (3, 5, 1030, False), (2, 3, 40001, False)])
def test_policy(b, t, v, placed, mean, name):
    say(f"policy b={b} t={t} v={v} placed={placed} {mean} {name}")
    check_policy(*make(b, t, v, DTYPES[name], v + t, placed, masked=b > 1), placed, mean)


def test_policy_with_token_advantages_and_without_a_reference():
    args = make(6, 20, 50, torch.float32, 1, True)
    check_policy(*args, True, "tokens", per_token=True)
    check_policy(*args, True, "orders", with_ref=False, coef=0.0)
    args = make(3, 4, 3001, torch.bfloat16, 1)
    check_policy(*args, False, "orders", per_token=True)
    check_policy(*args, False, "tokens", with_ref=False, coef=0.0)


@pytest.mark.parametrize("v", [20, 2000])
def test_policy_of_nothing_is_zero(v):
    logits, tokens, _ = make(3, 4, v, torch.float32)
    logits[:] = float("nan")
    z, k = dev(logits, tokens)
    ones = torch.ones(3, 4, device="cuda")
    for mean in ("tokens", "orders"):
        res = cc.cc_policy_loss(z, k, ones, ones[:, 0].contiguous(), ones, torch.zeros(3, 4, dtype=torch.bool, device="cuda"), mean=mean)
        assert (res.stats == 0).all() and (res.logprob == 0).all() and (res.grad_logits == 0).all()
    res = cc.cc_policy_loss(z[:0], k[:0], ones[:0], ones[:0, 0].contiguous())
    assert (res.stats == 0).all() and res.grad_logits.shape == (0, 4, v)


def test_policy_gradient_against_differences():
    """Both losses are in 32 bits: their difference is off by at most two of the loss's bounds, over twice the step."""
    b, t, v, eps = 6, 20, 20, 2.0 ** -5
    logits, tokens, mask = make(b, t, v, torch.float32, 3, True)
    _, _, lp, valid, rel = ref.rows(logits, tokens, mask, True, SCALE)
    old, other, adv = policy_inputs(lp, False)
    direction = torch.randn(logits.shape, generator=torch.Generator().manual_seed(2)) * 0.02
    args = dev(tokens, old, adv, other, mask)
    def run(z):
        return cc.cc_policy_loss(z.cuda(), *args, True, SCALE, 0.2, 0.25, 0.1)
    slope = float((run(logits).grad_logits.cpu().double() * direction).sum())
    up, down = run(logits + eps * direction), run(logits - eps * direction)
    estimate = (float(up.stats[0]) - float(down.stats[0])) / (2 * eps)
    total = float(ref.policy(lp, valid, old, other, adv, 0.2, 0.25, 0.1, "tokens")[3])
    noise = (total * (rel + 16 * U) + abs(float(up.stats[0])) * U) / eps
    assert float(up.stats[2]) == float(down.stats[2])           # no ratio crossed a border
    assert abs(estimate - slope) <= noise + 1e-2 * abs(slope)


# ------------------------------------------------------------------------------------------------------ preference


def check_preference(logits, tokens, mask, placed, with_ref=True, smoothing=0.1, beta=0.25):
    dtype = logits.dtype
    pairs = logits.shape[0] // 2
    p, rest, lp, valid, rel = ref.rows(logits, tokens, mask, placed, SCALE)
    other = (lp + 0.2 * torch.randn(lp.shape, generator=torch.Generator().manual_seed(4))).float() if with_ref else None
    if not with_ref:
        beta = 0.02
    beta32, smoothing32 = float(torch.tensor(beta)), float(torch.tensor(smoothing))
    loss, margin, slope = ref.preference(lp, valid, other, beta32, smoothing32)
    scale = 64.0 if dtype is torch.float16 else 1.0
    z, k, m, r = dev(logits, tokens, mask, other)
    res = cc.cc_preference_loss(z, k, r, m, placed, SCALE, beta, smoothing, grad_scale=scale)
    within(res.logprob, lp, finish(lp, lp.abs() * U + rel, torch.float32), "logprob")
    # a margin sums what each position may be off; the loss's derivative is at most 1, the slope's a quarter of beta / pairs
    per_order = (valid * rel).sum(1)
    margin_err = beta32 * (per_order[:pairs] + per_order[pairs:])
    within(res.margin, margin, finish(margin, margin_err + margin.abs() * U, torch.float32), "margin")
    within(res.loss, loss, finish(loss, margin_err.mean() + loss * U, torch.float32), "loss")
    slope_err = (beta32 / pairs * (margin_err / 4)).repeat(2).unsqueeze(1) + slope.abs() * U
    want = ref.grad_logits(p, rest, tokens, valid, slope * SCALE * scale)
    err = ref.grad_logits(p, -rest, tokens, valid, slope_err.expand_as(slope) * SCALE * scale).abs() + want.abs() * (2 * rel + 8 * U)
    within(res.grad_logits, want, finish(want, err, dtype), "gradient")
    again = cc.cc_preference_loss(z, k, r, m, placed, SCALE, beta, smoothing, grad_scale=scale)
    assert all(torch.equal(x, y) for x, y in zip(res, again))
    bare = cc.cc_preference_loss(z, k, r, m, placed, SCALE, beta, smoothing, grad=False)
    assert bare.grad_logits is None and torch.equal(bare.loss, res.loss) and torch.equal(bare.margin, res.margin)
    place = z.clone()
    cc.cc_preference_loss(place, k, r, m, placed, SCALE, beta, smoothing, grad_scale=scale, grad_logits=place)
    assert torch.equal(place, res.grad_logits)


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("b,t,v,placed", [(2, 1, 3, False), (4, 8, 8, True), (60, 4, 10, True), (6, 100, 100, True), (2, 30, 1000, True),
                                          (4, 7, 1500, False), (2, 3, 40001, False)])
def test_preference(b, t, v, placed, name):
    say(f"preference b={b} t={t} v={v} placed={placed} {name}")
    check_preference(*make(b, t, v, DTYPES[name], v + t, placed), placed)


def test_preference_without_a_reference_and_with_smoothing_at_its_ends():
    args = make(6, 20, 50, torch.float32, 1, True)
    check_preference(*args, True, with_ref=False)
    check_preference(*args, True, smoothing=0.0)
    check_preference(*args, True, smoothing=1.0)


def test_preference_of_nothing():
    z, k = dev(*make(4, 3, 50, torch.float32)[:2])
    none = torch.zeros(4, 3, dtype=torch.uint8, device="cuda")
    res = cc.cc_preference_loss(z, k, None, none)
    assert abs(float(res.loss) - 0.6931471805599453) < 1e-7 and (res.margin == 0).all() and (res.grad_logits == 0).all()
    res = cc.cc_preference_loss(z[:0], k[:0])
    assert float(res.loss) == 0 and res.margin.shape == (0,)
    res = cc.cc_preference_loss(z[:, :0], k[:, :0])
    assert abs(float(res.loss) - 0.6931471805599453) < 1e-7 and (res.margin == 0).all()


def test_a_preference_beyond_doubt():
    """Margins in the hundreds: the loss is the margin or nothing, and nothing overflows."""
    logits, tokens, _ = make(2, 200, 30, torch.float32, 5, masked=False)
    other = torch.zeros(2, 200)
    other[0] = -60.0
    for flip in (False, True):
        r = other.flip(0) if flip else other
        res = cc.cc_preference_loss(*dev(logits, tokens), r.cuda(), beta=1.0)
        assert torch.isfinite(res.loss) and torch.isfinite(res.grad_logits).all()
        assert (float(res.loss) == 0) != flip and abs(float(res.margin[0])) > 1000


def test_preference_gradient_against_differences():
    b, t, v, eps = 6, 20, 20, 2.0 ** -5
    logits, tokens, mask = make(b, t, v, torch.float32, 3, True)
    _, _, lp, valid, rel = ref.rows(logits, tokens, mask, True, SCALE)
    direction = torch.randn(logits.shape, generator=torch.Generator().manual_seed(2)) * 0.1
    k, m, r = dev(tokens, mask, (lp + 0.1).float())
    def run(z):
        return cc.cc_preference_loss(z.cuda(), k, r, m, True, SCALE, 0.25, 0.1)
    slope = float((run(logits).grad_logits.cpu().double() * direction).sum())
    up, down = float(run(logits + eps * direction).loss), float(run(logits - eps * direction).loss)
    per_order = (valid * rel).sum(1)
    noise = (0.25 * float((per_order[:3] + per_order[3:]).mean()) + abs(up) * U) / eps
    assert abs((up - down) / (2 * eps) - slope) <= noise + 1e-2 * abs(slope)


# ------------------------------------------------------------------------------------------------- undefined logits


def undefined_rows(v, dtype):
    """Orders of five rows: nothing but NaN; NaN beside minus infinity, the token one or the other; minus infinity alone; numbers."""
    logits, tokens, _ = make(2, 5, v, dtype, v, masked=False)
    nan, low = float("nan"), float("-inf")
    logits[0, 0] = nan
    logits[0, 1] = low
    logits[0, 1, v // 2] = nan
    tokens[0, 1] = v // 2
    logits[0, 2] = nan
    logits[0, 2, v // 3] = low
    tokens[0, 2] = v // 3
    logits[0, 3] = low
    return logits, tokens


@pytest.mark.parametrize("name", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("v", [2, 6, 64, 300, 1024, 1025, 5000, 140001])
def test_undefined_logits_are_not_taken_for_impossible_ones(v, name):
    say(f"undefined logits v={v} {name}")
    logits, tokens = undefined_rows(v, DTYPES[name])
    z, k = dev(logits, tokens)
    nan_rows = torch.tensor([[True, True, True, False, False], [False] * 5])
    lp, rows = cc.cc_token_logprob(z, k, None, False, SCALE)
    assert torch.equal(lp.isnan().cpu(), nan_rows) and float(lp[0, 3]) == float("-inf")
    clean = z.clone()
    clean[0, :3] = 1.0
    same, _ = cc.cc_token_logprob(clean, k, None, False, SCALE)
    assert torch.equal(lp[0, 3:], same[0, 3:]) and torch.equal(lp[1], same[1])
    slope = torch.ones(2, 5, device="cuda")
    grad = cc.cc_token_logprob_backward(z, k, None, False, SCALE, rows, slope)
    assert grad[0, :3].isnan().all() and (grad[0, 3] == 0).all() and torch.isfinite(grad[1]).all()
    place = z.clone()
    cc.cc_token_logprob_backward(place, k, None, False, SCALE, rows, slope, grad_logits=place)
    assert torch.equal(place.isnan(), grad.isnan()) and torch.equal(place.nan_to_num(), grad.nan_to_num())
    # no loss of an undefined model is a number, with an advantage or without
    old = torch.full((2, 5), -1.0, device="cuda")
    for advantage in (1.0, -1.0, 0.0):
        res = cc.cc_policy_loss(z, k, old, torch.full((2,), advantage, device="cuda"), scale=SCALE)
        assert res.stats[0].isnan() and res.grad_logits[0, :3].isnan().all() and torch.isfinite(res.grad_logits[1]).all()
    res = cc.cc_preference_loss(z, k, old, scale=SCALE)
    assert res.loss.isnan() and res.margin.isnan().all() and res.grad_logits[0, :3].isnan().all()


@pytest.mark.parametrize("v", [1, 8, 65, 1000])
@pytest.mark.parametrize("orders", [1, 40])
def test_an_undefined_last_candidate(v, orders):
    """The last rank of an order has one candidate: undefined, its log-probability and its gradient are, and nothing else is."""
    logits, tokens, _ = make(orders, v, v, torch.float32, v, placed=True, masked=False)
    say(f"undefined last candidate v={v} orders={orders}")
    last = tokens[0, -1].item()
    logits[0, -1] = float("nan")
    z, k = dev(logits, tokens)
    lp, rows = cc.cc_token_logprob(z, k, None, True, SCALE)
    hit = torch.zeros_like(lp, dtype=torch.bool)
    hit[0, -1] = True
    assert torch.equal(lp.isnan(), hit)
    grad = cc.cc_token_logprob_backward(z, k, None, True, SCALE, rows, torch.ones_like(lp))
    nan_at = torch.zeros_like(grad, dtype=torch.bool)
    nan_at[0, -1, last] = True
    assert torch.equal(grad.isnan(), nan_at) and (grad[0, -1][~nan_at[0, -1]] == 0).all()
    if v > 1:
        # two candidates, one of them impossible, the other undefined: both gradients are undefined
        before = tokens[0, -2].item()
        z[0, -2] = float("-inf")
        z[0, -2, last] = float("nan")
        lp, rows = cc.cc_token_logprob(z, k, None, True, SCALE)
        grad = cc.cc_token_logprob_backward(z, k, None, True, SCALE, rows, torch.ones_like(lp))
        nan_at[0, -2, last] = nan_at[0, -2, before] = True
        assert lp[0, -2].isnan() and torch.equal(grad.isnan(), nan_at)


@pytest.mark.parametrize("v,placed", [(6, True), (300, False), (300, True), (5000, False)])
def test_an_infinite_logit_makes_its_row_undefined(v, placed):
    say(f"infinite logit v={v} placed={placed}")
    logits, tokens, _ = make(3, 5, v, torch.float32, v, placed=placed, masked=False)
    if not placed:
        tokens[:] = torch.arange(5, dtype=torch.int32)
    logits[0, 1, tokens[0, 1]] = float("inf")                   # the token's own
    logits[1, 2, tokens[1, 4]] = float("inf")                   # another candidate's
    z, k = dev(logits, tokens)
    lp, rows = cc.cc_token_logprob(z, k, None, placed, SCALE)
    hit = torch.zeros(3, 5, dtype=torch.bool, device="cuda")
    hit[0, 1] = hit[1, 2] = True
    assert torch.equal(lp.isnan(), hit) and torch.isfinite(lp[~hit]).all()
    grad = cc.cc_token_logprob_backward(z, k, None, placed, SCALE, rows, torch.ones_like(lp))
    nan_at = hit.unsqueeze(2).expand_as(grad).clone()
    if placed:
        nan_at[0, 1, tokens[0, 0]] = nan_at[1, 2, tokens[1, 0]] = nan_at[1, 2, tokens[1, 1]] = False
    assert torch.equal(grad.isnan(), nan_at)


# ---------------------------------------------------------------------------------------- margins that are not finite


@pytest.mark.parametrize("pairs,t", [(2, 5), (5, 70), (1100, 3)])
@pytest.mark.parametrize("smoothing,impossible", [(0.0, "dearer"), (1.0, "cheaper")])
def test_an_infinite_margin_on_the_right_side_costs_nothing(pairs, t, smoothing, impossible):
    """A term of the loss whose coefficient is zero has no part in it, whatever the margin."""
    say(f"preference pairs={pairs} t={t} smoothing={smoothing} impossible={impossible}")
    v = 9
    logits, tokens, _ = make(2 * pairs, t, v, torch.float32, pairs, masked=False)
    order = 1 if impossible == "cheaper" else pairs + 1
    logits[order, 2, tokens[order, 2]] = float("-inf")
    z, k = dev(logits, tokens)
    res = cc.cc_preference_loss(z, k, scale=SCALE, beta=0.5, label_smoothing=smoothing)
    assert float(res.margin[1]) == float("-inf" if impossible == "cheaper" else "inf")
    others = [i for i in range(2 * pairs) if i % pairs != 1]
    rest = cc.cc_preference_loss(z[others].contiguous(), k[others].contiguous(), scale=SCALE, beta=0.5, label_smoothing=smoothing)
    want = float(rest.loss) * (pairs - 1) / pairs
    assert abs(float(res.loss) - want) <= 4 * U * want                      # two results' roundings, the product's and the quotient's
    assert (res.grad_logits[[1, pairs + 1]] == 0).all() and torch.isfinite(res.grad_logits).all()


def test_an_infinite_margin_on_the_wrong_side():
    logits, tokens, _ = make(4, 5, 9, torch.float32, 3, masked=False)
    logits[1, 2, tokens[1, 2]] = float("-inf")
    z, k = dev(logits, tokens)
    for smoothing in (0.0, 0.25):
        res = cc.cc_preference_loss(z, k, scale=SCALE, beta=0.5, label_smoothing=smoothing)
        assert float(res.margin[1]) == float("-inf") and float(res.loss) == float("inf") and torch.isfinite(res.grad_logits).all()
    # a margin that counts for nothing
    res = cc.cc_preference_loss(z, k, scale=SCALE, beta=0.0)
    assert (res.margin == 0).all() and abs(float(res.loss) - 0.6931471805599453) <= U and (res.grad_logits == 0).all()


def test_two_impossible_sequences_have_no_margin():
    logits, tokens, _ = make(4, 5, 9, torch.float32, 3, masked=False)
    logits[1, 2, tokens[1, 2]] = logits[3, 4, tokens[3, 4]] = float("-inf")
    res = cc.cc_preference_loss(*dev(logits, tokens), scale=SCALE, beta=0.5)
    assert res.margin[1].isnan() and torch.isfinite(res.margin[0]) and res.loss.isnan()
    assert torch.isfinite(res.grad_logits[[0, 2]]).all()


# ---------------------------------------------------------------------------------------------------- small divergences


@pytest.mark.parametrize("v,placed", [(8, False), (8, True), (700, False), (3000, False)])
@pytest.mark.parametrize("apart", [1e-7, 1e-6, 1e-4, 1e-3, 3e-2, 1.0, 20.0, -1e-6, -1e-3, -0.5, -30.0])
def test_the_divergence_of_policies_near_each_other(v, placed, apart):
    """Where all candidates' logits are equal the log-probability is -log of their number, to within 1e-12 (the series of the logarithm
    5e-13, 64-bit operations), and the divergence exp(x) - 1 - x of x = ref - lp moves by |exp(x) - 1| times that."""
    say(f"policy v={v} placed={placed} apart={apart}")
    b, t = 3, 4
    logits = torch.full((b, t, v), 0.5)
    tokens = torch.arange(t, dtype=torch.int32).expand(b, t).contiguous()
    lp = -torch.log(torch.tensor([float(v - (i if placed else 0)) for i in range(t)], dtype=torch.float64)).expand(b, t)
    other = (lp + apart).float()
    away = other.double() - lp
    grown = torch.expm1(away)
    kl = torch.where(away.abs() < 0.1, away ** 2 * (1 / 2 + away / 6 + away ** 2 / 24 + away ** 3 / 120 + away ** 4 / 720 + away ** 5 / 5040 + away ** 6 / 40320),
                     grown - away)
    coef = 1000.0
    args = dev(logits, tokens, lp.float(), torch.zeros(b), other)
    res = cc.cc_policy_loss(*args, placed=placed, scale=SCALE, kl_coef=coef)
    # the mean's weights and terms are rounded to 32 bits (a weight, a divergence, the coefficient's product, the result: 4 u)
    bound = 4 * U * float(kl.mean()) + float(grown.abs().mean()) * 1e-12
    assert abs(float(res.stats[1]) - float(kl.mean())) <= bound
    assert abs(float(res.stats[0]) - coef * float(kl.mean())) <= coef * (bound + 2 * U * float(kl.mean()))
    # the slope is -coef (exp(x) - 1) / 12, the token's gradient SCALE (1 - p) times that
    want = -coef * grown / (b * t) * SCALE * (1 - torch.exp(lp))
    got = res.grad_logits.gather(2, args[1].long().unsqueeze(2)).squeeze(2).cpu().double()
    err = coef * SCALE / (b * t) * torch.exp(away) * 1e-12 + want.abs() * 16 * U
    if placed:
        keep = lp < 0
        got, want, err = got[keep], want[keep], err[keep]
    assert ((got - want).abs() <= err).all()


@pytest.mark.parametrize("v", [30, 2000])
def test_the_divergence_of_an_impossible_token_is_infinite(v):
    logits, tokens, _ = make(2, 4, v, torch.float32, 8, masked=False)
    logits[0, 2, tokens[0, 2]] = float("-inf")
    z, k, old = dev(logits, tokens, torch.full((2, 4), -3.0))
    for coef in (0.0, 0.1):
        res = cc.cc_policy_loss(z, k, old, torch.ones(2, device="cuda"), old, scale=SCALE, kl_coef=coef)
        assert float(res.stats[1]) == float("inf")
        assert float(res.stats[0]) == float("inf") if coef else torch.isfinite(res.stats[0])


# ------------------------------------------------------------------------------- many orders, many pairs, longer rows

# Orders enough that a workgroup's wavefronts take several batches of rows each, and a last one that is not full: batches of 32 rows
# (up to 8 vectors of logits), 16, 8, 4 (up to 64), 2 and 1, two or four of them.
BATCHES = [(1024, 130, 3, False, "f32"), (1024, 130, 20, True, "f32"), (1030, 200, 40, False, "bf16"), (600, 270, 50, False, "f32"),
           (520, 150, 100, True, "f16"), (300, 130, 130, True, "f32"), (256, 150, 200, False, "f32"), (300, 100, 300, True, "bf16"),
           (520, 150, 120, True, "f32"), (64, 520, 300, False, "f32"), (64, 520, 520, True, "f16"), (32, 520, 600, False, "f32"), (20, 900, 1000, True, "f32")]


@pytest.fixture
def at_once(monkeypatch):
    """The definition for all positions together."""
    monkeypatch.setattr(ref, "rows", ref.rows_at_once)


def inputs(case):
    """The case's logits, tokens and mask; orders that are longer than their vocabulary place every node again and again."""
    b, t, v, placed, name = case
    logits, tokens, mask = make(b, t, v, DTYPES[name], t + v, placed and v >= t)
    if placed and v < t:
        again = [torch.rand(b, v, generator=torch.Generator().manual_seed(i)).argsort(1) for i in range(-(-t // v))]
        tokens = torch.cat(again, 1)[:, :t].to(torch.int32).contiguous()
    return logits, tokens, mask


@pytest.mark.parametrize("case", BATCHES, ids=str)
def test_logprob_of_many_batches(case, at_once):
    say(f"logprob {case}")
    check_logprob(*inputs(case), case[3])


@pytest.mark.parametrize("case", BATCHES, ids=str)
def test_policy_of_many_batches(case, at_once):
    say(f"policy {case}")
    check_policy(*inputs(case), case[3], "tokens" if case[1] % 4 else "orders", per_token=case[0] == 300)


@pytest.mark.parametrize("case", BATCHES, ids=str)
def test_preference_of_many_batches(case, at_once):
    say(f"preference {case}")
    check_preference(*inputs(case), case[3])


@pytest.mark.parametrize("mean", ["tokens", "orders"])
@pytest.mark.parametrize("b,t,v", [(1024, 1, 4), (1025, 3, 9), (3100, 5, 7), (1500, 70, 6), (2, 700, 5)])
def test_policy_of_more_orders_than_are_counted_at_once(b, t, v, mean, at_once):
    say(f"policy b={b} t={t} v={v} {mean}")
    check_policy(*make(b, t, v, torch.float32, b, masked=b > 2), False, mean)


@pytest.mark.parametrize("pairs,t", [(4, 65), (5, 65), (5, 1000), (64, 300), (4, 2048), (3, 2049), (1024, 64), (1025, 64), (1025, 3), (1300, 65), (66000, 1)])
def test_preference_of_many_pairs(pairs, t, at_once):
    say(f"preference pairs={pairs} t={t}")
    check_preference(*make(2 * pairs, t, 5, torch.float32, pairs + t), False)
    if pairs < 100:
        check_preference(*make(2 * pairs, t, 6, torch.bfloat16, pairs + t), False, smoothing=0.0, with_ref=False)


@pytest.mark.parametrize("b,t,v,name", [(2, 3, 5000, "bf16"), (2, 3, 9001, "f16"), (2, 3, 9001, "f32"), (2, 2, 20003, "bf16"), (1, 3, 32769, "f32"),
                                        (1, 3, 65536, "f32"), (2, 2, 65537, "f32"), (1, 3, 100003, "f32"), (2, 2, 65537, "f16"),
                                        (2, 2, 70001, "bf16"), (1, 3, 131072, "bf16"), (2, 2, 131073, "bf16"), (1, 3, 140007, "f16"),
                                        (1, 2, 300009, "bf16")])
def test_policy_of_longer_rows(b, t, v, name, at_once):
    """On both sides of what each kernel keeps of a row, and rows that none keeps: read again for the gradient, in place too."""
    say(f"policy b={b} t={t} v={v} {name}")
    check_policy(*make(b, t, v, DTYPES[name], v, masked=b > 1), False, "tokens")


def test_many_long_rows(at_once):
    """2048 rows and more that are longer than a workgroup's stride are taken by smaller workgroups: the same rows for all orders."""
    b, t, v = 64, 33, 16401
    say(f"logprob b={b} t={t} v={v}")
    logits, tokens, _ = make(1, t, v, torch.float32, 6, masked=False)
    p, rest, lp, valid, rel = ref.rows(logits, tokens, None, False, SCALE)
    z, k = logits.cuda().expand(b, t, v), tokens.cuda().expand(b, t).contiguous()
    got, rows = cc.cc_token_logprob(z, k, None, False, SCALE)
    within(got, lp.expand(b, t), finish(lp, lp.abs() * U + rel, torch.float32).expand(b, t), "logprob")
    slope = torch.randn(t, generator=torch.Generator().manual_seed(1))
    grad = cc.cc_token_logprob_backward(z, k, None, False, SCALE, rows, slope.cuda().expand(b, t).contiguous())
    want = ref.grad_logits(p, rest, tokens, valid, slope.double() * SCALE)
    assert torch.equal(grad, grad[:1].expand(b, t, v))
    within(grad[:1], want, finish(want, want.abs() * (2 * rel + 8 * U), torch.float32), "gradient")


@pytest.mark.parametrize("pairs,t", [(256, 64), (257, 63), (257, 64), (512, 32), (512, 33), (1024, 16), (1024, 17), (1025, 7)])
def test_preference_of_pairs_on_both_sides_of_one_workgroup(pairs, t, at_once):
    say(f"preference pairs={pairs} t={t}")
    check_preference(*make(2 * pairs, t, 5, torch.float32, pairs + t), False)


@pytest.mark.parametrize("b,t,v", [(16, 32, 4096), (16, 32, 4097), (7, 73, 4096), (7, 73, 4097), (16, 32, 32767), (16, 32, 32768), (7, 73, 32767),
                                   (16, 32, 16384), (16, 32, 16385), (89, 23, 16385), (64, 32, 16385), (64, 32, 32767), (64, 32, 32768)])
def test_rows_on_both_sides_of_larger_workgroups(b, t, v, at_once):
    """About 512 and 2048 rows, of one turn of the larger workgroups, four and eight: the same logits for all orders."""
    say(f"logprob b={b} t={t} v={v}")
    logits, tokens, _ = make(1, t, v, torch.float32, 6, masked=False)
    p, rest, lp, valid, rel = ref.rows(logits, tokens, None, False, SCALE)
    z, k = logits.cuda().expand(b, t, v), tokens.cuda().expand(b, t).contiguous()
    got, rows = cc.cc_token_logprob(z, k, None, False, SCALE)
    within(got, lp.expand(b, t), finish(lp, lp.abs() * U + rel, torch.float32).expand(b, t), "logprob")
    slope = torch.randn(t, generator=torch.Generator().manual_seed(1))
    grad = cc.cc_token_logprob_backward(z, k, None, False, SCALE, rows, slope.cuda().expand(b, t).contiguous())
    want = ref.grad_logits(p, rest, tokens, valid, slope.double() * SCALE)
    assert torch.equal(grad, grad[:1].expand(b, t, v))
    within(grad[:1], want, finish(want, want.abs() * (2 * rel + 8 * U), torch.float32), "gradient")


@pytest.mark.parametrize("v", [12, 2500])
def test_no_advantage_and_no_ratio(v):
    """A token that was impossible when it was drawn, and still is, has no ratio: without an advantage it has no part either."""
    logits, tokens, _ = make(2, 4, v, torch.float32, v, masked=False)
    logits[0, 1, tokens[0, 1]] = float("-inf")
    z, k = dev(logits, tokens)
    old, _ = cc.cc_token_logprob(z, k, scale=SCALE)
    res = cc.cc_policy_loss(z, k, old, torch.zeros(2, device="cuda"), scale=SCALE)
    assert float(old[0, 1]) == float("-inf") and (res.stats == 0).all() and (res.grad_logits == 0).all()
