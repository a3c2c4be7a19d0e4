"""The 64-bit reference of the order model against central differences and against itself, on the CPU."""
import pytest
import torch

import order_model_reference as ref


def rand(seed, *shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def differences(f, at, step=1e-5):
    """Central differences of a scalar function: their own error is of the order of step squared."""
    out = torch.zeros_like(at)
    for i in range(at.numel()):
        up, down = at.clone(), at.clone()
        up.view(-1)[i] += step
        down.view(-1)[i] -= step
        out.view(-1)[i] = (f(up) - f(down)) / (2 * step)
    return out


def test_embedding_gradient_is_the_lookup_s_adjoint():
    ids = torch.tensor([[0, 3, -1], [3, 7, 2]], dtype=torch.int32)
    table, weight = rand(1, 5, 4), rand(2, 2, 3, 4)
    got, _ = ref.embed_backward(weight, ids, 5, 0.5)
    assert torch.allclose(got, differences(lambda x: (ref.embed(x, ids, 0.5) * weight).sum(), table), atol=1e-8)


@pytest.mark.parametrize("lengths", [None, [4, 0, 7]])
def test_scan_gradients(lengths):
    b, t, d = 3, 7, 2
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    x, gate, h0, gh, gl = rand(1, b, t, d), rand(2, b, t, d), rand(3, b, d), rand(4, b, t, d), rand(5, b, d)

    def loss(x, gate, h0):
        h, last, _, _ = ref.scan(x, gate, h0, n)
        return (h * gh).sum() + (last * gl).sum()

    (dx, dg, dh0), _ = ref.scan_backward(x, gate, h0, n, gh, gl)
    assert torch.allclose(dx, differences(lambda v: loss(v, gate, h0), x), atol=1e-8)
    assert torch.allclose(dg, differences(lambda v: loss(x, v, h0), gate), atol=1e-8)
    assert torch.allclose(dh0, differences(lambda v: loss(x, gate, v), h0), atol=1e-8)


def token_case(placed):
    b, t, v = 4, 3, 5
    logits = rand(7, b, t, v)
    tokens = torch.stack([torch.randperm(v, generator=torch.Generator().manual_seed(i))[:t] for i in range(b)]).to(torch.int32)
    mask = torch.ones(b, t, dtype=torch.bool)
    mask[1, 0] = mask[2, 2] = False
    mask[3] = False
    return logits, tokens, mask


@pytest.mark.parametrize("placed", [False, True])
@pytest.mark.parametrize("mean", ["tokens", "orders"])
def test_policy_gradient(placed, mean):
    logits, tokens, mask = token_case(placed)
    old, other, adv = rand(8, 4, 3) * 0.3 - 1.5, rand(9, 4, 3) * 0.3 - 1.5, rand(10, 4)

    def loss(z):
        _, _, lp, valid, _ = ref.rows(z, tokens, mask, placed, 0.75)
        return ref.policy(lp, valid, old, other, adv, 0.2, 0.3, 0.1, mean)[0][0]

    p, rest, lp, valid, _ = ref.rows(logits, tokens, mask, placed, 0.75)
    slope = ref.policy(lp, valid, old, other, adv, 0.2, 0.3, 0.1, mean)[1]
    got = ref.grad_logits(p, rest, tokens, valid, slope * 0.75)
    assert torch.allclose(got, differences(loss, logits), atol=1e-8)
    assert (got[3] == 0).all() and (got[1, 0] == 0).all()


@pytest.mark.parametrize("placed", [False, True])
def test_preference_gradient(placed):
    logits, tokens, mask = token_case(placed)
    other = rand(9, 4, 3)

    def loss(z):
        _, _, lp, valid, _ = ref.rows(z, tokens, mask, placed, 1.25)
        return ref.preference(lp, valid, other, 0.4, 0.1)[0]

    p, rest, lp, valid, _ = ref.rows(logits, tokens, mask, placed, 1.25)
    slope = ref.preference(lp, valid, other, 0.4, 0.1)[2]
    assert torch.allclose(ref.grad_logits(p, rest, tokens, valid, slope * 1.25), differences(loss, logits), atol=1e-8)


def test_placed_probabilities_are_of_the_nodes_that_are_left():
    logits, tokens, _ = token_case(True)
    p, rest, lp, _, _ = ref.rows(logits, tokens, None, True, 1.0)
    for b in range(4):
        left = set(range(5))
        for t in range(3):
            assert {j for j in range(5) if p[b, t, j] > 0} == left
            left.remove(int(tokens[b, t]))
    assert torch.allclose(p.sum(2), torch.ones(4, 3, dtype=torch.float64))
    assert torch.allclose(torch.exp(lp), 1 - rest)


def test_bounds_catch_a_planted_mistake():
    """A state rounded to 16 bits after every step is outside the bounds that the kernels are held to."""
    x, gate, h0 = rand(1, 1, 40, 3), rand(2, 1, 40, 3) + 2, rand(3, 1, 3)
    h, _, err, _ = ref.scan(x, gate, h0, None)
    s, wrong = h0.clone(), torch.zeros_like(h)
    for i in range(40):
        s = (torch.sigmoid(gate[:, i]) * s + torch.sigmoid(-gate[:, i]) * x[:, i]).bfloat16().double()
        wrong[:, i] = s
    with pytest.raises(AssertionError):
        ref.within(wrong, h, ref.finish(h, err, torch.float32), "h")


@pytest.mark.parametrize("placed", [False, True])
def test_rows_at_once_are_rows(placed):
    g = torch.Generator().manual_seed(2)
    logits = 3 * torch.randn(4, 12, 15, generator=g)
    tokens = torch.randint(-1, 16, (4, 12), generator=g, dtype=torch.int32)
    mask = torch.rand(4, 12, generator=g) < 0.8
    logits[0, 1] = float("-inf")
    logits[1, 2, 3:] = float("-inf")
    logits[2, 5, 1] = 60.0
    tokens[2, 5], mask[0, 1], mask[1, 2], mask[2, 5] = 1, True, True, True
    one, other = ref.rows(logits, tokens, mask, placed, 0.75), ref.rows_at_once(logits, tokens, mask, placed, 0.75)
    for x, y in zip(one[:3], other[:3]):
        assert torch.allclose(x, y, rtol=1e-13, atol=1e-300)
    assert torch.equal(one[3], other[3]) and one[4] == other[4]
