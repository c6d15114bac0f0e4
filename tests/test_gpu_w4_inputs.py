"""4-bit experts on rows with a large common part, in every kernel of bf16 layers, and without x.

The products accumulate (16 + code) * x and take (16 + zero) * sum x off: with x = 20 + noise the two are up to 24 * 128 * 20 each and what
is left may be small.  The element-by-element bar of tests/test_gpu_w4.py is for any x (2^-16 of 31 * scale * sum |x|, beside the
rounding of the stored result); its bar of the mean is not used, as that one counts on rounding errors of a sum without a trend."""
import numpy as np
import pytest
import torch

from inputs import workloads as wl
from tests import test_gpu_w4 as base
from tests.helpers import BF16_U

pytestmark = pytest.mark.gpu


def _elementwise(got, want, terms, tops, dtype, what):
    bar = BF16_U * (1 + 2.0 ** -7) * np.abs(want) + 2.0 ** -16 * tops + 2.0 ** -17 * terms + 2.0 ** -20 * np.abs(want)
    excess = np.abs(got - want) - bar
    assert np.isfinite(got).all() and excess.max() <= 0.0, f"{what}: {excess.max():.3e} beyond the bar"


# K split over the waves; 16-row tiles, a shared sum split and with codes ahead; 32-row tiles with one and two units per wave
@pytest.mark.parametrize("shape", [(33, 256, 384, 8, 3, 2, 4), (20, 200, 648, 64, 4, 4, 4), (50, 648, 1032, 64, 4, 2, 4),
                                   (70, 648, 1032, 64, 4, 3, 4), (60, 136, 2008, 8, 1, 4, 2), (130, 264, 1928, 4, 2, 2, 2)])
@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, False), (128, True)])
def test_rows_with_a_common_part(shape, group, zeros, monkeypatch):
    layer, xd, _, _, values, tops, x = base.make(*shape, "bf16", group, zeros, seed=sum(shape), spread=0.5)
    x = wl.round_to_bf16((x + 20.0).astype(np.float32))
    xd.copy_(torch.from_numpy(x))
    layer.dispatch(xd)
    layer.expert_ffn_w4(xd)
    monkeypatch.setattr(base, "compare", _elementwise)
    base.check_network(layer, x.astype(np.float64), values, tops, "bf16", f"{shape} {group} {zeros}")


@pytest.mark.parametrize("shape", [(9, 136, 72, 4, 0, 2, 2), (60, 2008, 136, 8, 0, 4, 2)])
def test_without_shared_experts_x_is_not_read(shape):
    layer, xd, *_ = base.make(*shape, "bf16", 64, True, seed=5)
    ref = layer.expert_ffn_w4(xd)[0].clone()
    layer.epd_y.fill_(7.0)
    assert torch.equal(layer.expert_ffn_w4(None)[0], ref)
