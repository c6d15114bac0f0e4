"""The backward pass with three rows per workgroup and row group, the last pass a part of one: more tokens than two passes of the grid
take, in every layout that a row length selects, with and without means and biases.  Bars: those of tests/test_gpu_block_norm.py
(at most 9 rows per row group)."""
import pytest
import torch

from paper_2505_13345_amd import binding as B
from tests.test_gpu_block_norm import case, check

pytestmark = pytest.mark.gpu


# waves per row 1, 2, 3, 4, 5, 8; two and four vectors per lane, where parameters and rows are read again in every pass
@pytest.mark.parametrize("kind,dtype,T,d", [
    ("layer", "bf16", 4201, 264), ("layer", "f32", 2101, 264), ("layer", "bf16", 1601, 1032), ("layer", "bf16", 1101, 2048),
    ("layer", "f32", 1103, 1032), ("rms", "f32", 1103, 1032), ("rms", "bf16", 1601, 1032), ("layer", "f32", 531, 2048),
    ("layer", "bf16", 531, 4104), ("rms", "bf16", 531, 4104), ("rms", "bf16", 531, 16384), ("layer", "bf16", 521, 16384),
    ("rms", "f32", 521, 8192), ("layer", "f32", 521, 8192)])
def test_three_passes(kind, dtype, T, d):
    check(*case(T, d, dtype, kind, kind, "channel", seed=d + T), f"{kind} {dtype} T={T} d={d}")


@pytest.mark.parametrize("post,pre,gate,dtype,T,d", [
    ("rms", "layer", "token", "bf16", 1101, 2048), ("layer", "rms", "element", "bf16", 531, 4104), (None, "layer", "token", "f32", 521, 8192),
    ("rms", None, "token", "bf16", 531, 16384)])
def test_three_passes_of_other_kinds(post, pre, gate, dtype, T, d):
    check(*case(T, d, dtype, post, pre, gate, seed=d + T), f"{post} {pre} {gate} {dtype} T={T} d={d}")


@pytest.mark.parametrize("kind,T,d", [("rms", 70, 264), ("layer", 1101, 2048), ("rms", 531, 16384)])
def test_without_dx(kind, T, d):
    norm, t, p, *_ = case(T, d, "bf16", kind, kind, "channel", seed=d)
    out, _ = norm.forward(t["x"], t["y"], **p)
    ref = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
    desc = B.make_block_norm(*norm._fixed, **p)
    dy = torch.full_like(ref["dy"], 7.0)
    sums = {n: torch.full_like(ref[n], 7.0) for n in ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias", "dgate")}
    B.occult_block_norm_backward(norm.cfg, desc, t["y"], out, t["dout"], t["dh"], None, dy, ws=norm.ws, **sums)
    for n, v in dict(sums, dy=dy).items():
        assert torch.equal(v, ref[n]), n
