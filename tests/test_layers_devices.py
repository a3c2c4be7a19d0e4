"""The norm's, the 8-bit rows' and products' and the shaping's calls refuse each tensor, and a stream, of another device than the current one: a
kernel launched here would read what may not be there.  Host only: tensors say that they are on a device, and the library is replaced."""
import types

import pytest
import torch

import paper_2105_14088_amd as cc
from paper_2105_14088_amd import binding, order_model


class Placed(torch.Tensor):
    """A tensor in host memory that says it is on a device (0 unless it is told another)."""
    at = 0
    is_cuda = True

    def get_device(self):
        return self.at


def tensor(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Placed)


def elsewhere(t):
    t = t.clone()
    t.at = 1
    return t


class Library:
    """Every call succeeds, every workspace has 256 bytes."""

    def __getattr__(self, name):
        return lambda *args: 256 if name.endswith("_workspace_bytes") else 0


I8, I32 = torch.int8, torch.int32
# each call with all the tensors that it takes
CALLS = {
    "cc_rms_norm": dict(x=tensor(3, 8), weight=tensor(8), residual=tensor(3, 8), out=tensor(3, 8), sum=tensor(3, 8), q=tensor(3, 8, dtype=I8),
                        scale=tensor(3), rstd=tensor(3)),
    "cc_rms_norm_backward": dict(grad_out=tensor(3, 8), h=tensor(3, 8), rstd=tensor(3), weight=tensor(8), grad_sum=tensor(3, 8), grad_h=tensor(3, 8),
                                 grad_weight=tensor(8), workspace=tensor(256, dtype=torch.uint8)),
    "cc_quantize_rows": dict(x=tensor(3, 8), q=tensor(3, 8, dtype=I8), scale=tensor(3)),
    "cc_product_i8": dict(x=tensor(3, 8, dtype=I8), x_scale=tensor(3), w=tensor(5, 8, dtype=I8), w_scale=tensor(5), bias=tensor(5), out=tensor(3, 5),
                          workspace=tensor(256, dtype=torch.uint8)),
    "cc_shape_logits": dict(logits=tensor(2, 3, 40), history=tensor(2, 7, dtype=I32), lengths=tensor(2, dtype=I32), penalties=tensor(2, 3),
                            starts=tensor(2, dtype=I32), bias=tensor(2, 40), allowed=tensor(2, 3, 2, dtype=I32), out=tensor(2, 3, 40)),
    "cc_shape_logits_backward": dict(grad_out=tensor(2, 3, 40), logits=tensor(2, 3, 40), history=tensor(2, 7, dtype=I32), lengths=tensor(2, dtype=I32),
                                     penalties=tensor(2, 3), starts=tensor(2, dtype=I32), bias=tensor(2, 40), allowed=tensor(2, 3, 2, dtype=I32),
                                     grad_logits=tensor(2, 3, 40)),
}


@pytest.fixture(autouse=True)
def on_device_0(monkeypatch):
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_current_raw_stream", lambda device: 100 + device)
    monkeypatch.setattr(order_model, "_several_devices", lambda: True, raising=False)
    monkeypatch.setattr(order_model, "lib", lambda: Library())
    order_model._norm_bytes.cache_clear()
    order_model._product_bytes.cache_clear()
    yield
    order_model._norm_bytes.cache_clear()
    order_model._product_bytes.cache_clear()


@pytest.mark.parametrize("call", CALLS)
def test_tensors_of_the_current_device_are_taken(call):
    getattr(cc, call)(**CALLS[call])
    getattr(cc, call)(**CALLS[call], stream=types.SimpleNamespace(cuda_stream=5, device_index=0))


@pytest.mark.parametrize("call,name", [(call, name) for call, args in CALLS.items() for name in args])
def test_each_tensor_of_another_device_is_refused(call, name):
    with pytest.raises(ValueError, match="current device"):
        getattr(cc, call)(**{**CALLS[call], name: elsewhere(CALLS[call][name])})


@pytest.mark.parametrize("call", CALLS)
def test_a_stream_of_another_device_is_refused(call):
    with pytest.raises(ValueError, match="current device"):
        getattr(cc, call)(**CALLS[call], stream=types.SimpleNamespace(cuda_stream=5, device_index=1))


@pytest.mark.parametrize("count", [1, 2])
def test_other_devices_are_looked_for_where_there_are_some(count, monkeypatch):
    monkeypatch.undo()
    monkeypatch.setattr(torch.cuda, "device_count", lambda: count)
    order_model._several_devices.cache_clear()
    assert order_model._several_devices() is (count == 2)
    order_model._several_devices.cache_clear()
