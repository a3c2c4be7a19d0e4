"""What the order model's calls refuse, on the host, before anything is launched."""
import ctypes

import pytest
import torch

import paper_2105_14088_amd as cc

pytestmark = pytest.mark.usefixtures("built_library")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
FAKE, ODD, NULL = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001), ctypes.c_void_p(0)
BIG = 1 << 40


def embed(**over):
    a = dict(table=FAKE, dtype=0, V=10, D=8, table_stride=8, ids=FAKE, n=4, scale=1.0, out=FAKE, out_stride=8)
    a.update(over)
    return cc.lib().cc_embed(*a.values(), NULL)


def embed_backward(**over):
    a = dict(grad=FAKE, dtype=2, n=4, D=8, grad_stride=8, ids=FAKE, V=10, scale=1.0, grad_table=FAKE, grad_dtype=2,
             grad_table_stride=8, accumulate=0, workspace=FAKE, workspace_bytes=BIG)
    a.update(over)
    return cc.lib().cc_embed_backward(*a.values(), NULL)


@pytest.mark.parametrize("over", [dict(table=NULL), dict(table=ODD), dict(ids=NULL), dict(ids=ODD), dict(out=NULL), dict(out=ODD),
                                  dict(dtype=3), dict(dtype=-1), dict(V=0), dict(V=1 << 30), dict(D=0), dict(D=(1 << 24) + 1), dict(n=-1),
                                  dict(n=1 << 30), dict(out_stride=7), dict(table_stride=-1), dict(scale=float("nan")),
                                  dict(scale=float("inf")), dict(dtype=1, out=ODD)])
def test_embed_refuses(over):
    assert embed(**over) == INVALID


def test_embed_of_nothing_is_nothing():
    assert embed(n=0, table=NULL, ids=NULL, out=NULL) == OK
    assert embed_backward(n=0, accumulate=1, grad=NULL, ids=NULL, grad_table=NULL, workspace=NULL, workspace_bytes=0) == OK


@pytest.mark.parametrize("over", [dict(grad=NULL), dict(grad=ODD), dict(ids=NULL), dict(grad_table=NULL), dict(grad_table=ODD), dict(dtype=3),
                                  dict(grad_dtype=1), dict(dtype=1, grad_dtype=2), dict(grad_table_stride=7), dict(V=0), dict(D=0),
                                  dict(n=-1), dict(scale=float("nan")), dict(grad_dtype=0, grad_table=ctypes.c_void_p(0x1002))])
def test_embed_backward_refuses(over):
    assert embed_backward(**over) == INVALID


def test_workspaces_are_asked_for():
    L = cc.lib()
    need = L.cc_embed_workspace_bytes(10, 8, 4)
    assert need > 0 and need % 256 == 0
    assert embed_backward(workspace=NULL) == WORKSPACE
    assert embed_backward(workspace_bytes=need - 1) == WORKSPACE
    assert embed_backward(workspace=ctypes.c_void_p(0x1010)) == WORKSPACE
    assert L.cc_embed_workspace_bytes(0, 8, 4) == 0 and L.cc_embed_workspace_bytes(10, 8, -1) == 0
    assert L.cc_gated_scan_workspace_bytes(2, 65536, 64) > 0 and L.cc_gated_scan_workspace_bytes(2, 1, 64) == 0
    assert L.cc_gated_scan_workspace_bytes(-1, 4, 4) == 0
    assert L.cc_token_workspace_bytes(3, 5) > 0 and L.cc_token_workspace_bytes(-1, 5) == 0
    assert scan(B=2, T=65536, D=64, h_stride_b=65536 * 64, h_stride_t=64, workspace=NULL) == WORKSPACE
    assert policy(workspace=NULL) == WORKSPACE and policy(workspace_bytes=1) == WORKSPACE
    assert preference(workspace=NULL) == WORKSPACE


def scan(**over):
    a = dict(x=FAKE, x_stride_b=32, x_stride_t=8, gate=FAKE, gate_stride_b=32, gate_stride_t=8, dtype=0, B=2, T=4, D=8,
             lengths=NULL, h0=NULL, h=FAKE, h_stride_b=32, h_stride_t=8, last=NULL, states=NULL, workspace=NULL, workspace_bytes=0)
    a.update(over)
    return cc.lib().cc_gated_scan(*a.values(), NULL)


def scan_backward(**over):
    a = dict(x=FAKE, x_stride_b=32, x_stride_t=8, gate=FAKE, gate_stride_b=32, gate_stride_t=8, dtype=0, B=2, T=4, D=8,
             lengths=NULL, states=FAKE, grad_h=FAKE, grad_h_stride_b=32, grad_h_stride_t=8, grad_last=NULL, grad_x=FAKE,
             grad_x_stride_b=32, grad_x_stride_t=8, grad_gate=FAKE, grad_gate_stride_b=32, grad_gate_stride_t=8, grad_h0=NULL,
             workspace=NULL, workspace_bytes=0)
    a.update(over)
    return cc.lib().cc_gated_scan_backward(*a.values(), NULL)


@pytest.mark.parametrize("over", [dict(x=NULL), dict(gate=NULL), dict(h=NULL), dict(x=ODD), dict(h0=ODD), dict(last=ODD), dict(states=ODD),
                                  dict(lengths=ODD), dict(dtype=7), dict(B=-1), dict(T=-1), dict(D=0), dict(D=1 << 25), dict(T=1 << 31),
                                  dict(B=1 << 20, T=1 << 20), dict(x_stride_t=-8), dict(h_stride_t=7), dict(h_stride_b=31)])
def test_scan_refuses(over):
    assert scan(**over) == INVALID


@pytest.mark.parametrize("over", [dict(states=NULL), dict(grad_h=NULL), dict(grad_x=NULL), dict(grad_gate=NULL), dict(grad_gate=ODD),
                                  dict(grad_last=ODD), dict(grad_h0=ODD), dict(grad_x_stride_b=31), dict(grad_gate_stride_t=0),
                                  dict(grad_h_stride_b=-1), dict(dtype=3)])
def test_scan_backward_refuses(over):
    assert scan_backward(**over) == INVALID


def test_scan_of_no_sequence_is_nothing():
    assert scan(B=0, x=NULL, gate=NULL, h=NULL) == OK
    assert scan_backward(B=0, x=NULL, gate=NULL, grad_h=NULL, grad_x=NULL, grad_gate=NULL, states=NULL) == OK


def logits_args(over):
    a = dict(logits=FAKE, dtype=0, B=2, T=4, V=16, stride_b=64, stride_t=16, tokens=FAKE, mask=NULL, placed=0, scale=1.0)
    a.update({k: over.pop(k) for k in list(over) if k in a})
    return list(a.values())


def logprob(**over):
    head = logits_args(over)
    a = dict(logprob=FAKE, rows=NULL)
    a.update(over)
    return cc.lib().cc_token_logprob(*head, *a.values(), NULL)


def logprob_backward(**over):
    head = logits_args(over)
    a = dict(rows=FAKE, grad_logprob=FAKE, grad_scale=1.0, grad_logits=FAKE, gsb=64, gst=16)
    a.update(over)
    return cc.lib().cc_token_logprob_backward(*head, *a.values(), NULL)


def policy(**over):
    head = logits_args(over)
    a = dict(old=FAKE, ref=NULL, advantage=FAKE, per_token=0, clip_low=0.2, clip_high=0.2, kl_coef=0.1, mean=0, grad_scale=1.0, stats=FAKE,
             logprob=FAKE, grad_logits=NULL, gsb=0, gst=0, workspace=FAKE, workspace_bytes=BIG)
    a.update(over)
    return cc.lib().cc_policy_loss(*head, *a.values(), NULL)


def preference(**over):
    head = logits_args(over)
    a = dict(ref=NULL, beta=0.1, smoothing=0.0, grad_scale=1.0, loss=FAKE, margin=FAKE, logprob=FAKE, grad_logits=NULL, gsb=0, gst=0,
             workspace=FAKE, workspace_bytes=BIG)
    a.update(over)
    return cc.lib().cc_preference_loss(*head, *a.values(), NULL)


@pytest.mark.parametrize("call", [logprob, logprob_backward, policy, preference])
@pytest.mark.parametrize("over", [dict(logits=NULL), dict(logits=ODD), dict(tokens=NULL), dict(tokens=ODD), dict(dtype=3), dict(V=0),
                                  dict(V=(1 << 24) + 1), dict(B=-2), dict(T=-1), dict(B=1 << 20, T=1 << 12), dict(stride_b=-1), dict(scale=0.0),
                                  dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(logprob=NULL)])
def test_calls_on_logits_refuse(call, over):
    if call is logprob_backward and "logprob" in over:
        over = dict(grad_logprob=NULL)
    assert call(**dict(over)) == INVALID


@pytest.mark.parametrize("call", [logprob, logprob_backward, policy, preference])
def test_placed_is_for_orders(call):
    assert call(placed=1, V=1025, stride_t=1025, stride_b=4100, **({"gsb": 4100, "gst": 1025} if call is logprob_backward else {})) == UNSUPPORTED
    assert call(placed=1, T=1025, stride_b=16400, **({"gsb": 16400} if call is logprob_backward else {})) == UNSUPPORTED


@pytest.mark.parametrize("over", [dict(grad_logits=NULL), dict(grad_logits=ODD), dict(gst=15), dict(gsb=63), dict(rows=NULL),
                                  dict(rows=ctypes.c_void_p(0x1004)), dict(grad_scale=float("inf")),
                                  dict(stride_b=64, stride_t=16, gsb=128)])       # in place with other strides
def test_logprob_backward_refuses(over):
    assert logprob_backward(**over) == INVALID


@pytest.mark.parametrize("over", [dict(old=NULL), dict(old=ODD), dict(ref=ODD), dict(advantage=NULL), dict(stats=NULL), dict(clip_low=-0.1),
                                  dict(clip_low=1.5), dict(clip_high=-1.0), dict(clip_high=float("inf")), dict(kl_coef=float("nan")),
                                  dict(mean=2), dict(grad_scale=float("nan")), dict(grad_logits=ODD), dict(grad_logits=FAKE, gsb=64, gst=8)])
def test_policy_refuses(over):
    assert policy(**over) == INVALID


@pytest.mark.parametrize("over", [dict(B=3), dict(beta=float("inf")), dict(smoothing=-0.1), dict(smoothing=1.1), dict(loss=NULL), dict(margin=NULL),
                                  dict(ref=ODD), dict(grad_scale=float("inf"))])
def test_preference_refuses(over):
    assert preference(**over) == INVALID


def test_no_position_needs_no_pointer():
    assert logprob(B=0, logits=NULL, tokens=NULL, logprob=NULL) == OK
    assert logprob_backward(T=0, logits=NULL, tokens=NULL, rows=NULL, grad_logprob=NULL, grad_logits=NULL) == OK


def test_binding_refuses_what_it_cannot_describe():
    t = torch.zeros(2, 3, 4)
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_embed(torch.zeros(4, 4), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="float32, float16 or bfloat16"):
        cc.cc_embed(torch.zeros(4, 4, dtype=torch.float64), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="B, T, D"):
        cc.cc_gated_scan(t[0], t[0])
    with pytest.raises(ValueError, match="B, T, V"):
        cc.cc_token_logprob(t[0], torch.zeros(3, 4, dtype=torch.int32))
    with pytest.raises(ValueError, match="GPU"):
        cc.cc_token_logprob(t, torch.zeros(2, 3, dtype=torch.int32))
    with pytest.raises(ValueError, match="accumulate"):
        cc.cc_embed_backward(_OnDevice(t), torch.zeros(2, 3, dtype=torch.int32), 5, accumulate=True)


class _OnDevice:
    """A tensor that says it is on the GPU: what the binding checks next is reached without one."""
    def __init__(self, t):
        self.t = t

    is_cuda = True

    def __getattr__(self, name):
        return getattr(self.t, name)
