"""The definitions that the kernels of the norm, the products in 8 bits and the shaped logits are tested against, by hand and by differences."""
import math

import pytest
import torch

import layers_reference as ref


def test_norm_by_hand():
    h = torch.tensor([[3.0, 4.0], [0.0, 0.0]])
    out, r = ref.norm(h, torch.tensor([1.0, 2.0]), 1e-30)
    assert torch.allclose(out[0], torch.tensor([3.0, 8.0]).double() / math.sqrt(12.5)) and out[1].abs().max() == 0
    q, scale = ref.eight_bits(h.double() * torch.tensor([1.0, 2.0]).double(), r)
    assert q[0].tolist() == [48.0, 127.0] and q[1].tolist() == [0.0, 0.0]
    assert float(scale[0]) == pytest.approx(8 / math.sqrt(12.5) / 127) and float(scale[1]) == 0


def test_eight_bits_at_borders_and_undefined():
    q, scale = ref.eight_bits(torch.tensor([[2.0, 1.0, -1.0], [math.inf, 1.0, 0.0], [math.nan, 1.0, 0.0]]).double(), torch.ones(3).double())
    assert q.tolist() == [[127.0, 64.0, -64.0], [0.0, 0.0, 0.0], [0.0, 0.0, 0.0]]      # 63.5: the even neighbour
    assert float(scale[0]) == 2 / 127 and torch.isnan(scale[1:]).all()


@pytest.mark.parametrize("with_weight", [True, False])
def test_norm_backward_by_differences(with_weight):
    g = torch.Generator().manual_seed(1)
    h = torch.randn(3, 7, generator=g, dtype=torch.float64)
    w = torch.randn(7, generator=g, dtype=torch.float64) if with_weight else None
    go, gs = torch.randn(3, 7, generator=g, dtype=torch.float64), torch.randn(3, 7, generator=g, dtype=torch.float64)
    eps, step = 1e-3, 1e-6

    def loss(hh, ww):
        return (ref.norm(hh, ww, eps)[0] * go).sum() + (hh * gs).sum()

    grad_h, grad_w = ref.norm_backward(go, h, w, ref.norm(h, w, eps)[1], gs)
    for i in range(3):
        for j in range(7):
            d = torch.zeros_like(h)
            d[i, j] = step
            assert float(loss(h + d, w) - loss(h - d, w)) / (2 * step) == pytest.approx(float(grad_h[i, j]), abs=1e-7)
    if with_weight:
        for j in range(7):
            d = torch.zeros_like(w)
            d[j] = step
            assert float(loss(h, w + d) - loss(h, w - d)) / (2 * step) == pytest.approx(float(grad_w[j]), abs=1e-7)


def test_product_by_hand():
    x = torch.tensor([[1, -2, 127]], dtype=torch.int8)
    w = torch.tensor([[3, 0, 1], [-128, 5, 2]], dtype=torch.int8)
    out = ref.product(x, torch.tensor([0.5]), w, torch.tensor([2.0, 4.0]), torch.tensor([1.0, 0.0]))
    assert out.tolist() == [[131.0, 2.0 * (-128 - 10 + 254)]]


def test_shaped_by_hand():
    z = torch.tensor([[[2.0, -2.0, 1.0, 5.0], [2.0, -2.0, 1.0, 5.0]]])
    history = torch.tensor([[0, 1, 0, 9, 2]], dtype=torch.int32)
    out, slope, _ = ref.shaped(z, history, torch.tensor([3]), torch.tensor([[2.0, 0.5, 0.25]]), torch.tensor([1]), torch.tensor([0.0, 0.0, 1.0, -math.inf]))
    # row 0 sees 0, 1, 0 and counts 1, 0; row 1 sees the padding 9 as well
    assert out[0, 0].tolist() == [1.0 - 0.75, -4.0 - 0.75, 2.0, -math.inf] and torch.equal(out[0, 0], out[0, 1])
    assert slope[0, 0].tolist() == [0.5, 2.0, 1.0, 0.0]
    out, _, _ = ref.shaped(z, history, torch.tensor([4]), torch.tensor([[1.0, math.inf, 0.0]]), allowed=torch.tensor([[[0b1011], [0b1111]]]))
    assert out[0].tolist() == [[-math.inf, -math.inf, -math.inf, 5.0], [-math.inf, -math.inf, -math.inf, 5.0]]
