"""One BlockNorm that serves several callers: a call that another thread makes between a call's checks and its launch must not change
what the first one launches."""
import pytest
import torch

from tests.test_gpu_block_norm import case

pytestmark = pytest.mark.gpu


class _Library:
    """The library, with another call made just before the next launch."""

    def __init__(self, lib, other):
        self._lib, self._other = lib, other

    def __getattr__(self, name):
        call = getattr(self._lib, name)

        def launch(*args):
            other, self._other = self._other, None
            if other:
                other()
            return call(*args)

        return launch


def test_parameters_of_a_call_are_its_own():
    norm, t, p, *_ = case(9, 264, "bf16", "rms", "layer", "channel", seed=21)
    others = {n: v * 2 + 1 for n, v in p.items()}
    out, h = (v.clone() for v in norm.forward(t["x"], t["y"], **p))
    ref = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items() if v is not None}
    lib = norm._lib
    elsewhere = torch.empty_like(out), torch.empty_like(out)
    norm._lib = _Library(lib, lambda: norm.forward(t["x"], t["y"], out=elsewhere[0], h=elsewhere[1], **others))
    got, got_h = norm.forward(t["x"], t["y"], **p)
    assert torch.equal(got, out) and torch.equal(got_h, h)
    assert not torch.equal(elsewhere[0], out)
    norm._lib = _Library(lib, lambda: norm.forward(t["x"], t["y"], out=elsewhere[0], h=elsewhere[1], **others))
    g = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
    for n, v in ref.items():
        assert torch.equal(g[n], v), n
