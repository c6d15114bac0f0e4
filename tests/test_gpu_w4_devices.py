"""Calls on 4-bit weights refuse another current device than the layer's, and tensors of another device than its buffers."""
import pytest
import torch

from tests.test_gpu_w4 import make

pytestmark = pytest.mark.gpu


class _Elsewhere:
    """A tensor of another device, as far as the checks look at it."""

    def __init__(self, t):
        self._t = t

    def __getattr__(self, name):
        return getattr(self._t, name)

    def get_device(self):
        return self._t.get_device() + 1


def test_refusals_of_other_devices(monkeypatch):
    layer, xd, logits, q, *_ = make(5, 64, 96, 4, 1, 2, 2, "bf16", 32, True)
    w = layer.dequantize_weights(q)
    there = lambda ts: tuple(_Elsewhere(t) for t in ts)
    for call in (lambda: layer.expert_ffn_w4(_Elsewhere(xd)), lambda: layer.forward_w4(logits, _Elsewhere(xd)),
                 lambda: layer.forward_w4(_Elsewhere(logits), xd), lambda: layer.quantize_weights(*there(w)),
                 lambda: layer.dequantize_weights(q._replace(codes=there(q.codes))),
                 lambda: layer.pack_weights_w4(q._replace(scales=there(q.scales))),
                 lambda: layer.pack_weights_w4(q._replace(zeros=there(q.zeros)))):
        with pytest.raises(ValueError, match="buffers are on cuda:0"):
            call()
    # x and the current device agree, and the layer is elsewhere
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: layer.expert_ffn_w4(_Elsewhere(xd)), lambda: layer.forward_w4(logits, _Elsewhere(xd)),
                 lambda: layer.quantize_weights(*w), lambda: layer.dequantize_weights(q), lambda: layer.pack_weights_w4(q)):
        with pytest.raises(ValueError, match="current device"):
            call()
