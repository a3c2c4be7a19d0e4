"""What the norm, the rows and products in 8 bits and the shaping of logits refuse, on the host, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2105_14088_amd as cc

pytestmark = pytest.mark.usefixtures("built_library")

OK, INVALID, WORKSPACE = 0, -1, -3
FAKE, OTHER, THIRD, ODD, NULL = (ctypes.c_void_p(v) for v in (0x1000, 0x2000, 0x3000, 0x1001, 0))
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")


def norm(**over):
    a = dict(x=FAKE, x_stride=8, residual=OTHER, residual_stride=8, dtype=2, n=4, D=8, weight=FAKE, weight_dtype=0, eps=1e-6, sum=THIRD, sum_stride=8,
             out=THIRD, out_stride=8, q=ODD, q_stride=8, scale=FAKE, rstd=FAKE)
    a.update(over)
    return cc.lib().cc_rms_norm(*a.values(), NULL)


def backward(**over):
    a = dict(grad_out=FAKE, grad_out_stride=8, h=OTHER, h_stride=8, dtype=2, n=4, D=8, weight=FAKE, weight_dtype=0, rstd=FAKE, grad_sum=NULL,
             grad_sum_stride=0, grad_h=THIRD, grad_h_stride=8, grad_weight=FAKE, grad_weight_dtype=0, accumulate=0, workspace=FAKE, workspace_bytes=BIG)
    a.update(over)
    return cc.lib().cc_rms_norm_backward(*a.values(), NULL)


def quantize(**over):
    a = dict(x=FAKE, x_stride=8, dtype=2, n=4, D=8, q=ODD, q_stride=8, scale=FAKE)
    a.update(over)
    return cc.lib().cc_quantize_rows(*a.values(), NULL)


def product(**over):
    a = dict(x=ODD, x_stride=8, x_scale=FAKE, w=ODD, w_stride=8, w_scale=FAKE, bias=NULL, M=4, N=6, K=8, out=FAKE, out_stride=6, dtype=2, workspace=FAKE,
             workspace_bytes=BIG)
    a.update(over)
    return cc.lib().cc_product_i8(*a.values(), NULL)


SHARED = dict(logits=FAKE, dtype=0, B=2, T=4, V=16, stride_b=64, stride_t=16, history=FAKE, L=5, history_stride=5, lengths=FAKE, starts=FAKE, penalties=FAKE,
              bias=FAKE, bias_stride=0, allowed=FAKE, allowed_stride_b=4, allowed_stride_t=1, out=OTHER, osb=64, ost=16)


def shape(**over):
    return cc.lib().cc_shape_logits(*{**SHARED, **over}.values(), NULL)


def shape_backward(**over):
    head = dict(grad=THIRD, gsb=64, gst=16)
    head.update({k: over.pop(k) for k in list(over) if k in head})
    return cc.lib().cc_shape_logits_backward(*head.values(), *{**SHARED, **over}.values(), NULL)


@pytest.mark.parametrize("over", [dict(x=NULL), dict(x=ODD), dict(residual=ODD), dict(weight=ODD), dict(weight=ctypes.c_void_p(0x1002)), dict(sum=ODD),
                                  dict(out=ODD), dict(scale=ODD), dict(rstd=ODD), dict(dtype=3), dict(dtype=-1), dict(weight_dtype=1), dict(n=-1),
                                  dict(n=1 << 31), dict(D=0), dict(D=(1 << 24) + 1), dict(x_stride=-1), dict(residual_stride=-8), dict(sum_stride=7),
                                  dict(out_stride=7), dict(q_stride=7), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(q=NULL),
                                  dict(scale=NULL), dict(sum=FAKE, sum_stride=9), dict(sum=OTHER, sum_stride=9)])
def test_norm_refuses(over):
    assert norm(**over) == INVALID


@pytest.mark.parametrize("over", [dict(grad_out=NULL), dict(grad_out=ODD), dict(h=NULL), dict(h=ODD), dict(rstd=NULL), dict(rstd=ODD), dict(weight=ODD),
                                  dict(grad_sum=ODD), dict(grad_h=NULL), dict(grad_h=ODD), dict(grad_weight=ODD), dict(grad_weight_dtype=1),
                                  dict(grad_weight_dtype=2), dict(weight=NULL), dict(dtype=3), dict(weight_dtype=1), dict(n=-1), dict(D=0),
                                  dict(D=1 << 25), dict(h_stride=-1), dict(grad_out_stride=-1), dict(grad_sum_stride=-1), dict(grad_h_stride=7),
                                  dict(grad_h=FAKE, grad_h_stride=9), dict(grad_sum=THIRD, grad_sum_stride=9)])
def test_norm_backward_refuses(over):
    assert backward(**over) == INVALID


@pytest.mark.parametrize("over", [dict(x=NULL), dict(x=ODD), dict(q=NULL), dict(scale=NULL), dict(scale=ODD), dict(dtype=3), dict(n=-1), dict(D=0),
                                  dict(D=1 << 25), dict(x_stride=-1), dict(q_stride=7)])
def test_quantize_refuses(over):
    assert quantize(**over) == INVALID


@pytest.mark.parametrize("over", [dict(x=NULL), dict(w=NULL), dict(x_scale=NULL), dict(x_scale=ODD), dict(w_scale=NULL), dict(w_scale=ODD), dict(bias=ODD),
                                  dict(out=NULL), dict(out=ODD), dict(dtype=3), dict(M=-1), dict(N=-1), dict(K=-1), dict(K=131072), dict(N=(1 << 24) + 1),
                                  dict(M=1 << 31), dict(M=1 << 30, N=1 << 20, out_stride=1 << 20), dict(x_stride=-1), dict(w_stride=-1), dict(out_stride=5)])
def test_product_refuses(over):
    assert product(**over) == INVALID


@pytest.mark.parametrize("call", [shape, shape_backward])
@pytest.mark.parametrize("over", [dict(logits=NULL), dict(logits=ODD), dict(dtype=3), dict(B=-1), dict(T=-1), dict(V=0), dict(V=(1 << 24) + 1),
                                  dict(B=1 << 20, T=1 << 12), dict(stride_b=-1), dict(stride_t=-1), dict(history=NULL), dict(history=ODD), dict(L=-1),
                                  dict(L=1 << 31), dict(history_stride=-1), dict(lengths=ODD), dict(starts=ODD), dict(penalties=ODD), dict(bias=ODD),
                                  dict(bias_stride=-1), dict(allowed=ODD), dict(allowed_stride_b=-1), dict(allowed_stride_t=-1), dict(out=NULL),
                                  dict(out=ODD), dict(osb=63), dict(ost=15)])
def test_shaping_refuses(call, over):
    assert call(**dict(over)) == INVALID


def test_in_place_only_where_it_was():
    assert shape(out=FAKE, osb=128) == INVALID and shape(out=FAKE, ost=32, osb=128) == INVALID
    assert shape_backward(out=THIRD, osb=128) == INVALID
    assert shape_backward(grad=NULL) == INVALID and shape_backward(grad=ODD) == INVALID and shape_backward(gsb=-1) == INVALID


def test_nothing_needs_no_pointer():
    assert norm(n=0, x=NULL, residual=NULL, weight=NULL, sum=NULL, out=NULL, q=NULL, scale=NULL, rstd=NULL) == OK
    assert backward(n=0, grad_out=NULL, h=NULL, rstd=NULL, grad_h=NULL, weight=NULL, grad_weight=NULL, workspace=NULL, workspace_bytes=0) == OK
    assert quantize(n=0, x=NULL, q=NULL, scale=NULL) == OK
    assert product(M=0, x=NULL, x_scale=NULL, w=NULL, w_scale=NULL, out=NULL) == OK and product(N=0, out=NULL) == OK
    assert shape(B=0, logits=NULL, out=NULL) == OK and shape_backward(T=0, logits=NULL, out=NULL, grad=NULL) == OK


def test_workspaces_are_asked_for():
    L = cc.lib()
    need = L.cc_rms_norm_workspace_bytes(4, 8)
    assert need > 0 and need % 256 == 0
    assert backward(workspace=NULL) == WORKSPACE and backward(workspace_bytes=need - 1) == WORKSPACE
    assert backward(workspace=ctypes.c_void_p(0x1010)) == WORKSPACE
    assert L.cc_rms_norm_workspace_bytes(-1, 8) == 0 and L.cc_rms_norm_workspace_bytes(4, 0) == 0
    assert L.cc_product_i8_workspace_bytes(-1, 4, 4) == 0 and L.cc_product_i8_workspace_bytes(4, 4, 1 << 17) == 0


def test_binding_refuses_what_it_cannot_describe():
    x, w = torch.zeros(3, 4), torch.zeros(4)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_rms_norm(x, w)
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        cc.cc_rms_norm(x.double(), w)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_rms_norm_backward(x, x, w[:3], w)
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        cc.cc_quantize_rows(x.to(torch.int8))
    with pytest.raises(ValueError, match="one length"):
        cc.cc_product_i8(torch.zeros(3, 4, dtype=torch.int8), x[:, 0], torch.zeros(2, 5, dtype=torch.int8), x[0, :2])
    with pytest.raises(ValueError, match="dtype"):
        cc.cc_product_i8(torch.zeros(3, 4, dtype=torch.int8), x[:, 0], torch.zeros(2, 4, dtype=torch.int8), x[0, :2], dtype=torch.int8)
    with pytest.raises(ValueError, match="B, T, V"):
        cc.cc_shape_logits(x)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_shape_logits(x[None])


def test_tensors_of_another_device_are_refused(monkeypatch):
    import types

    from paper_2105_14088_amd import binding, order_model
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: 100 + device)
    assert order_model._stream_at(types.SimpleNamespace(get_device=lambda: 0), None) == 100
    with pytest.raises(ValueError, match="current device"):
        order_model._stream_at(types.SimpleNamespace(get_device=lambda: 1), None)
    with pytest.raises(ValueError, match="current device"):
        order_model._stream_at(types.SimpleNamespace(get_device=lambda: 1), types.SimpleNamespace(cuda_stream=5))
