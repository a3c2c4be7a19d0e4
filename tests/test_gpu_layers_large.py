"""Offsets that pass 32 bits: the last rows of large calls against calls on these rows alone."""
import pytest
import torch

import paper_2105_14088_amd as cc
from gpu_util import say

pytestmark = [pytest.mark.gpu, pytest.mark.usefixtures("built_library")]


def filled(*shape, dtype, seed=0):
    """A pattern that no two near rows share, made in pieces."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    flat = t.view(-1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    piece = torch.randn(1 << 22, generator=g, device="cuda")
    for at in range(0, flat.numel(), piece.numel()):
        part = flat[at:at + piece.numel()]
        part.copy_((piece[:part.numel()] * (1 + at % 7)).to(dtype) if dtype.is_floating_point else (piece[:part.numel()] * 30).clamp(-127, 127).to(dtype))
    return t


def test_norm_and_rows():
    n, d = 70000, 33000
    say(f"large norm {n} {d}")
    x = filled(n, d, dtype=torch.bfloat16)
    w = torch.randn(d, device="cuda")
    res = cc.cc_rms_norm(x, w, quantized=True, save_rstd=True)
    q, scale = cc.cc_quantize_rows(x)
    for part in (slice(0, 3), slice(n - 5, n)):
        want = cc.cc_rms_norm(x[part].contiguous(), w, quantized=True, save_rstd=True)
        assert torch.equal(res.out[part], want.out) and torch.equal(res.q[part], want.q) and torch.equal(res.rstd[part], want.rstd)
        wq, ws = cc.cc_quantize_rows(x[part].contiguous())
        assert torch.equal(q[part], wq) and torch.equal(scale[part], ws)
    grad_h, _ = cc.cc_rms_norm_backward(res.out, x, res.rstd)
    want, _ = cc.cc_rms_norm_backward(res.out[-5:], x[-5:], res.rstd[-5:])
    assert torch.equal(grad_h[-5:], want)


def test_norm_of_registers():
    n, d = 1200000, 2048
    say(f"large norm {n} {d}")
    x = filled(n, d, dtype=torch.bfloat16)
    res = cc.cc_rms_norm(x, quantized=True, save_rstd=True)
    want = cc.cc_rms_norm(x[-7:], quantized=True, save_rstd=True)
    assert torch.equal(res.out[-7:], want.out) and torch.equal(res.q[-7:], want.q)
    grad_h, _ = cc.cc_rms_norm_backward(res.out, x, res.rstd)
    assert torch.equal(grad_h[-7:], cc.cc_rms_norm_backward(res.out[-7:], x[-7:], res.rstd[-7:])[0])


@pytest.mark.parametrize("m,n,k", [(70000, 33000, 32), (20, 140000, 32768), (300000, 8, 16000)])
def test_product(m, n, k):
    say(f"large product {m} {n} {k}")
    x, w = filled(m, k, dtype=torch.int8), filled(n, k, dtype=torch.int8, seed=1)
    xs, ws = torch.rand(m, device="cuda"), torch.rand(n, device="cuda")
    out = cc.cc_product_i8(x, xs, w, ws)
    rows, channels = min(m, 40), min(n, 50)
    want = cc.cc_product_i8(x[m - rows:], xs[m - rows:], w[n - channels:], ws[n - channels:])
    assert torch.equal(out[m - rows:, n - channels:], want)


@pytest.mark.parametrize("b,t,v", [(1, 36000, 65536), (2200, 1000, 1000)])
def test_shape(b, t, v):
    say(f"large shape {b} {t} {v}")
    z = filled(b, t, v, dtype=torch.bfloat16)
    history = torch.randint(0, v, (b, 64), device="cuda", dtype=torch.int32)
    penalties = torch.tensor([1.5, 0.5, 0.25], device="cuda").repeat(b, 1)
    out = cc.cc_shape_logits(z, history, None, penalties)
    lengths = torch.full((1,), t - 3, dtype=torch.int32, device="cuda")
    want = cc.cc_shape_logits(z[-1:, -3:], history[-1:], lengths, penalties[-1:])
    assert torch.equal(out[-1:, -3:], want)
    back = cc.cc_shape_logits_backward(out, z, history, None, penalties)
    assert torch.equal(back[-1:, -3:], cc.cc_shape_logits_backward(out[-1:, -3:], z[-1:, -3:], history[-1:], lengths, penalties[-1:]))
