"""The gradient of the pre norm alone, h = N_pre(x), from a description whose x_scale is not 1; and of a residual sum whose dy is not
wanted, which has x_scale.  Bars: those of tests/test_gpu_block_norm.py."""
import pytest
import torch

from oracle import block_norm as bn
from paper_2505_13345_amd import binding as B
from paper_2505_13345_amd.norm import BlockNorm
from tests.test_gpu_block_norm import GRADIENT_BAR, SUM_BAR, case, close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("T,d", [(1, 64), (37, 264), (21, 2056)])
@pytest.mark.parametrize("stream", [False, True])
def test_gradient_of_the_pre_norm_alone(dtype, kind, T, d, stream):
    norm, t, p, th, ph, cfg = case(T, d, dtype, None, kind, None, seed=d)
    assert cfg["x_scale"] != 1.0
    norm.forward(t["x"], **p)
    g = norm.backward(t["x"], t["dout"] if stream else None, t["dh"], **p)
    want = bn.gradients(th["x"], None, th["dout"] if stream else None, th["dh"], cfg, ph)
    for n, w in want.items():
        close(g[n], w, GRADIENT_BAR if n == "dx" else SUM_BAR, n)
    assert g["dy"] is None
    # the same bits as from a description without a residual scale
    first = {n: v.clone() for n, v in g.items() if v is not None}
    one = BlockNorm(T, d, dtype, None, kind, pre_eps=cfg["pre_eps"], weight_offset=cfg["offset"])
    again = one.backward(t["x"], t["dout"] if stream else None, t["dh"], **p)
    for n, v in first.items():
        assert torch.equal(v, again[n]), n


def test_residual_sum_whose_dy_is_not_wanted():
    """The same buffers, but there was a y: dx has the residual scale, whether or not y is handed over."""
    norm, t, p, th, ph, cfg = case(21, 264, "bf16", None, "rms", None, seed=3)
    out, _ = norm.forward(t["x"], t["y"], **p)
    full = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
    close(full["dx"], bn.gradients(out.cpu().double().numpy(), th["y"], th["dout"], th["dh"], cfg, ph)["dx"], GRADIENT_BAR, "dx")
    dx = full["dx"].clone()
    for kw in (dict(want_dy=False), dict(y=t["y"], want_dy=False), dict(want_dy=True)):
        g = norm.backward(out, t["dout"], t["dh"], **kw, **p)
        assert torch.equal(g["dx"], dx) and (g["dy"] is None) == (not kw["want_dy"]), kw


def test_frozen_block_behind_a_post_norm_or_a_gate():
    """dy not wanted, y not handed over, in descriptions that the pre norm alone cannot have: x_scale is in dx."""
    for post, gate in (("rms", None), (None, "channel")):
        norm, t, p, th, ph, cfg = case(9, 264, "f32", post, "rms", gate, seed=5)
        out, _ = norm.forward(t["x"], t["y"], **p)
        dx = norm.backward(out, t["dout"], t["dh"], t["y"], **p)["dx"].clone()
        desc = B.make_block_norm(*norm._fixed, **p)
        got = torch.full_like(dx, 7.0)
        B.occult_block_norm_backward(norm.cfg, desc, None, out, t["dout"], t["dh"], got, None)
        assert torch.equal(got, dx), (post, gate)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_residual_sum_without_any_norm(dtype):
    """out = x_scale * x + y_scale * y: without a pre norm there is no form without y, so x_scale is in dx whatever is handed over."""
    norm, t, p, *_ = case(9, 264, dtype, None, None, None, seed=6)
    out, _ = norm.forward(t["x"], t["y"])
    ref = norm.backward(out, t["dout"], y=t["y"])["dx"].clone()
    assert torch.equal(ref, (t["dout"].float() * 0.75).to(ref.dtype))
    for kw in (dict(), dict(want_dy=False), dict(want_dy=True)):
        assert torch.equal(norm.backward(out, t["dout"], **kw)["dx"], ref), kw
