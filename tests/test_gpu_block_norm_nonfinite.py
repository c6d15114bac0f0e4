"""Infinities and NaN that a gradient's formula does not read, or that belong to other rows."""
import pytest
import torch

from tests.test_gpu_block_norm import case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("gate", [None, "channel", "token", "element"])
def test_dy_without_a_post_norm_does_not_depend_on_y(dtype, pre, gate):
    """Without a post norm dy = y_scale * gate * D: no value of y is in it."""
    norm, t, p, *_ = case(9, 264, dtype, None, pre, gate, seed=41)
    out, _ = norm.forward(t["x"], t["y"], **p)
    out = out.clone()
    ref = norm.backward(out, t["dout"], t["dh"] if pre else None, t["y"], **p)["dy"].clone()
    t["y"][2, 5], t["y"][5, 9], t["y"][7] = float("inf"), float("nan"), float("-inf")
    got = norm.backward(out, t["dout"], t["dh"] if pre else None, t["y"], **p)["dy"]
    assert torch.equal(got, ref)


@pytest.mark.parametrize("T,d", [(1, 64), (5, 264), (3, 1032)])
def test_an_infinite_gate_of_the_first_token(T, d):
    """Its terms are infinite and those of the other tokens finite, so the sums over tokens are infinite, with the sign of its term:
    the lanes behind the last token, which have no token, add nothing."""
    norm, t, p, *_ = case(T, d, "bf16", "layer", "rms", "token", seed=43)
    out, _ = norm.forward(t["x"], t["y"], **p)
    out = out.clone()
    p["gate"][0] = float("inf")
    g = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
    term = -1.5 / 0.75 * g["dx"][0].float()      # y_scale * D, from dx = x_scale * D
    assert (term != 0).all()
    assert torch.equal(g["dpost_bias"], torch.sign(term) * float("inf"))
