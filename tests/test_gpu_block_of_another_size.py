"""forward_block refuses a norm made for other rows than the layer's: the calls beneath see addresses and totals only."""
import pytest
import torch

from paper_2505_13345_amd.norm import BlockNorm
from tests.test_gpu_w4 import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,dtype", [(12, 64, "bf16"), (3, 128, "bf16"), (6, 64, "f32"), (5, 64, "bf16")])
def test_norm_of_another_size(T, d, dtype):
    layer, xd, *_ = make(6, 64, 96, 4, 1, 2, 2, "bf16", 32, True)
    w_router = torch.zeros((4, 64), dtype=torch.bfloat16, device=layer.device)
    h = torch.zeros_like(xd)
    with pytest.raises(ValueError, match="norm is for"):
        layer.forward_block(xd, h, w_router, BlockNorm(T, d, dtype))
