"""The norms around a block (occult_block_norm and its backward pass) against the float64 oracle.

Bars.  A stored bf16 value is off by one rounding, BF16_U of its value (f32: 2^-24).  The float32 arithmetic before it: a row's sums
add at most 8 * 4 values per lane, then 6 lane exchanges and 8 waves (46 additions), and a term passes fewer than 16 further
operations, so every term of a result is off by less than 64 * 2^-24 = 2^-18 of its magnitude; a gradient of a norm multiplies
three such sums, hence 2^-16; sums over tokens add fewer than 600 times here (at most 9 rows per row group, 512
groups of a workgroup, 16 + 16 workgroups), hence 2^-14.  The oracle returns the sum of the magnitudes of each result's terms,
and the bars are relative to that."""
import numpy as np
import pytest
import torch

from oracle import block_norm as bn
from paper_2505_13345_amd import binding as B
from paper_2505_13345_amd.norm import BlockNorm
from tests.helpers import BF16_U, require_gpu, say

pytestmark = pytest.mark.gpu

FORWARD_BAR, GRADIENT_BAR, SUM_BAR = 2.0 ** -18, 2.0 ** -16, 2.0 ** -14


def case(T, d, dtype, post, pre, gate, params=("post_weight", "post_bias", "pre_weight", "pre_bias"), seed=0, offset=1.0):
    """Tensors on the GPU, the same values in float64 on the host, and the oracle's description."""
    dev = require_gpu()
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    gen = torch.Generator().manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=gen).to(dt)
    t = {"x": normal(T, d) * 2, "y": normal(T, d) + 0.5, "dout": normal(T, d), "dh": normal(T, d)}
    p = {n: normal(d) * 0.3 for n in params if {"post": post, "pre": pre}[n.split("_")[0]]}
    if gate:
        p["gate"] = normal(*{"channel": (d,), "token": (T,), "element": (T, d)}[gate])
    cfg = dict(post=post, pre=pre, gate=gate, x_scale=0.75, y_scale=-1.5, post_eps=1e-5, pre_eps=1e-6, offset=offset)
    norm = BlockNorm(T, d, dtype, post, pre, gate, cfg["x_scale"], cfg["y_scale"], cfg["post_eps"], cfg["pre_eps"], offset)
    return norm, {n: v.to(dev) for n, v in t.items()}, {n: v.to(dev) for n, v in p.items()}, host(t), host(p), cfg


def host(tensors):
    return {n: v.detach().cpu().double().numpy() for n, v in tensors.items()}


def unit(dtype):
    return BF16_U if dtype in ("bf16", torch.bfloat16) else 2.0 ** -24


def close(got, want, bar, what):
    value, scale = want
    u = unit(got.dtype)
    diff = np.abs(got.detach().cpu().double().numpy() - value)
    excess = diff - (u * (1 + 2.0 ** -7) * np.abs(value) + bar * scale + 1e-37)
    assert np.isfinite(diff).all() and excess.max() <= 0.0, f"{what}: {excess.max():.3e} beyond the bar"


def check(norm, t, p, th, ph, cfg, what):
    say(what)
    out, h = norm.forward(t["x"], t["y"], **p)
    close(out, bn.stream(th["x"], th["y"], cfg, ph), FORWARD_BAR, what + " out")
    stored = host({"out": out})["out"]
    if cfg["pre"]:
        close(h, bn.pre_norm(stored, cfg, ph), FORWARD_BAR, what + " h")
    else:
        assert h is None
    g = norm.backward(out, t["dout"], t["dh"] if cfg["pre"] else None, t["y"], **p)
    want = bn.gradients(stored, th["y"], th["dout"], th["dh"], cfg, ph)
    assert {n for n, v in g.items() if v is not None} == set(want)
    for n, w in want.items():
        summed = g[n].dim() == 1 and n != "dgate" or (n == "dgate" and cfg["gate"] != "element")
        close(g[n], w, SUM_BAR if summed else GRADIENT_BAR, f"{what} {n}")
    return out, h, g


# rows of one vector, of part of a wave, of several vectors per lane, of several waves; odd numbers of vectors
@pytest.mark.parametrize("d", [8, 64, 72, 264, 520, 1000, 1032, 1536, 1600, 2048, 2056, 2560, 2568, 4104, 8192, 16384])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_row_lengths(d, kind):
    for T in (1, 3, 70):
        check(*case(T, d, "bf16", kind, kind, "channel", seed=d + T), f"d={d} T={T} {kind}")


@pytest.mark.parametrize("d", [4, 36, 260, 516, 1028, 2044, 4096, 8192])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_row_lengths_f32(d, kind):
    for T in (1, 5, 33):
        check(*case(T, d, "f32", kind, kind, "channel", seed=d + T), f"f32 d={d} T={T} {kind}")


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("gate", [None, "channel", "token", "element"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kinds(post, pre, gate, dtype):
    check(*case(19, 264, dtype, post, pre, gate, seed=1), f"{post} {pre} {gate} {dtype}")


@pytest.mark.parametrize("params", [(), ("post_weight",), ("post_bias", "pre_weight"), ("pre_bias",)])
@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_parameters_left_out(params, offset):
    check(*case(9, 520, "bf16", "rms", "layer", None, params, seed=2, offset=offset), f"{params} {offset}")
    check(*case(9, 520, "bf16", "rms", "rms", "token", params, seed=2, offset=offset), f"{params} {offset} rms")


@pytest.mark.parametrize("T,d", [(2100, 2048), (2100, 72), (1500, 4104)])
def test_many_tokens(T, d):
    for gate in ("channel", "element"):
        check(*case(T, d, "bf16", "rms", "rms", gate, seed=5), f"T={T} d={d} {gate}")


def test_more_rows_than_one_pass_of_the_grid():
    """Forward: beyond 4096 workgroups.  The last rows and a sample of the others."""
    dev = require_gpu()
    T, d = 16384 + 37, 2048
    norm, t, p, *_ = case(1, d, "bf16", "rms", "rms", "channel")
    big = BlockNorm(T, d, "bf16", "rms", "rms", "channel", 0.75, -1.5, 1e-5, 1e-6, 1.0)
    gen = torch.Generator(device=dev).manual_seed(3)
    x, y = (torch.randn((T, d), device=dev, generator=gen).to(torch.bfloat16) for _ in range(2))
    out, h = big.forward(x, y, **p)
    for i in list(range(0, T, 1111)) + [T - 1]:
        one, one_h = norm.forward(x[i:i + 1], y[i:i + 1], **p)
        assert torch.equal(one[0], out[i]) and torch.equal(one_h[0], h[i]), i   # a token's results do not depend on T


def test_rows_beyond_4_gib():
    """Buffers of 4.4 GB: the first, middle and last rows against a call on those rows alone (a token's bits do not depend on T)."""
    dev = require_gpu()
    T, d = 270_000, 8192
    pick = [0, 1, T // 2, 262_143, 262_144, T - 1]
    gen = torch.Generator(device=dev).manual_seed(4)
    x, y, dout, dh = (torch.randn((T, d), device=dev, generator=gen, dtype=torch.bfloat16) for _ in range(4))
    w = torch.randn(d, device=dev, generator=gen, dtype=torch.bfloat16)
    big, small = BlockNorm(T, d, post="rms", pre="rms"), BlockNorm(len(pick), d, post="rms", pre="rms")
    out, h = big.forward(x, y, post_weight=w, pre_weight=w)
    some, some_h = small.forward(x[pick], y[pick], post_weight=w, pre_weight=w)
    assert torch.equal(out[pick], some) and torch.equal(h[pick], some_h)
    g = big.backward(out, dout, dh, y, post_weight=w, pre_weight=w)
    part = small.backward(some, dout[pick], dh[pick], y[pick], post_weight=w, pre_weight=w)
    assert torch.equal(g["dx"][pick], part["dx"]) and torch.equal(g["dy"][pick], part["dy"])


def test_pre_norm_alone():
    norm, t, p, th, ph, cfg = case(21, 1000, "bf16", None, "rms", None)
    same, h = norm.forward(t["x"], **p)
    assert same is t["x"]
    close(h, bn.pre_norm(th["x"], cfg, ph), FORWARD_BAR, "h")
    g = norm.backward(t["x"], None, t["dh"], **p)
    want = bn.gradients(th["x"], None, None, th["dh"], dict(cfg, x_scale=0.75), ph)
    for n in ("dx", "dpre_weight", "dpre_bias"):
        close(g[n], want[n], SUM_BAR if n != "dx" else GRADIENT_BAR, n)
    assert g["dy"] is None


def test_plain_residual_sum_without_kept_y():
    norm, t, p, th, ph, cfg = case(21, 264, "bf16", None, "rms", None)
    out, _ = norm.forward(t["x"], t["y"], **p)
    with_y = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items() if v is not None}
    without = norm.backward(out, t["dout"], t["dh"], want_dy=True, **p)
    for n, v in with_y.items():
        assert torch.equal(v, without[n]), n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_zeros_and_extreme_rows(dtype):
    """A row of zeros has no direction (the norm is 0 and its gradient q / sqrt(eps)); rows of tiny and of large values."""
    norm, t, p, th, ph, cfg = case(6, 264, dtype, "rms", "layer", "token", seed=7)
    for name in ("x", "y"):
        t[name][1] = 0
        t[name][2] *= 1e-15
        t[name][3] *= 1e15
        th[name] = host({"a": t[name]})["a"]
    check(norm, t, p, th, ph, cfg, f"zeros {dtype}")


def test_infinities_and_nan_stay_in_their_rows():
    norm, t, p, *_ = case(8, 520, "bf16", "rms", "rms", "token", seed=8)
    out, h = (v.clone() for v in norm.forward(t["x"], t["y"], **p))
    g = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items()}
    t["x"][2, 5], t["y"][5, 9] = float("inf"), float("nan")
    out2, h2 = norm.forward(t["x"], t["y"], **p)
    g2 = norm.backward(out2, t["dout"], t["dh"], t["y"], **p)
    keep = [0, 1, 3, 4, 6, 7]
    for a, b in ((out, out2), (h, h2), (g["dx"], g2["dx"]), (g["dy"], g2["dy"]), (g["dgate"], g2["dgate"])):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(out2[5]).all() and torch.isinf(out2[2, 5])


def test_in_place():
    norm, t, p, *_ = case(37, 2056, "bf16", "rms", "rms", "channel", seed=9)
    out, h = (v.clone() for v in norm.forward(t["x"], t["y"], **p))
    ref = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items() if v is not None}
    x, y = t["x"].clone(), t["y"].clone()
    norm.forward(x, y, out=x, h=y, **p)
    assert torch.equal(x, out) and torch.equal(y, h)
    desc = B.make_block_norm(*norm._fixed, **p)
    dout, y = t["dout"].clone(), t["y"].clone()
    B.occult_block_norm_backward(norm.cfg, desc, y, out, dout, t["dh"], dout, y)
    assert torch.equal(dout, ref["dx"]) and torch.equal(y, ref["dy"])


def test_accumulated_gradients():
    norm, t, p, *_ = case(130, 264, "f32", "layer", "layer", "channel", seed=10)
    out, _ = norm.forward(t["x"], t["y"], **p)
    sums = ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias", "dgate")
    once = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items()}
    twice = norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=True, **p)
    for n in sums:
        assert torch.equal(twice[n], once[n] + once[n]), n
    for n in ("dx", "dy"):
        assert torch.equal(twice[n], once[n]), n


def test_token_gate_gradient_is_not_accumulated_and_the_same_every_time():
    norm, t, p, *_ = case(2100, 1032, "bf16", "rms", "rms", "token", seed=11)
    out, _ = norm.forward(t["x"], t["y"], **p)
    a = {n: v.clone() for n, v in norm.backward(out, t["dout"], t["dh"], t["y"], **p).items() if v is not None}
    b = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
    for n, v in a.items():
        assert torch.equal(v, b[n]), n
    c = norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=True, **p)
    assert torch.equal(c["dgate"], a["dgate"])


def test_nothing_behind_the_last_row_is_written():
    dev = require_gpu()
    T, d = 5, 264
    norm, t, p, *_ = case(T, d, "bf16", "rms", "rms", "channel", seed=12)
    pad = {n: torch.full((T + 4, d), 7.0, dtype=torch.bfloat16, device=dev) for n in ("out", "h", "dx", "dy")}
    ws = torch.full((B.occult_block_norm_backward_ws_bytes(norm.cfg, B.make_block_norm(*norm._fixed, **p)) // 4 + 64,), 7.0, device=dev)
    dw = torch.full((d + 8,), 7.0, device=dev)
    desc = B.make_block_norm(*norm._fixed, **p)
    B.occult_block_norm(norm.cfg, desc, t["x"], t["y"], pad["out"], pad["h"])
    B.occult_block_norm_backward(norm.cfg, desc, t["y"], pad["out"], t["dout"], t["dh"], pad["dx"], pad["dy"], dpost_weight=dw, ws=ws)
    for n, v in pad.items():
        assert (v[T:] == 7.0).all(), n
    assert (dw[d:] == 7.0).all() and (ws[-64:] == 7.0).all()


def test_no_tokens():
    dev = require_gpu()
    norm = BlockNorm(0, 64, "bf16", "rms", "rms")
    w = torch.ones(64, dtype=torch.bfloat16, device=dev)
    empty = torch.zeros((0, 64), dtype=torch.bfloat16, device=dev)
    out, h = norm.forward(empty, empty, post_weight=w)
    assert out.shape == (0, 64) and h.shape == (0, 64)
    dw = torch.full((64,), 7.0, device=dev)
    desc = B.make_block_norm(*norm._fixed, post_weight=w)
    B.occult_block_norm_backward(norm.cfg, desc, None, None, None, None, None, None, dpost_weight=dw, accumulate=True)
    assert (dw == 7.0).all()
    B.occult_block_norm_backward(norm.cfg, desc, None, None, None, None, None, None, dpost_weight=dw)
    assert (dw == 0.0).all()


def test_refusals_of_the_buffers():
    norm, t, p, *_ = case(4, 64, "bf16", "rms", "rms", "channel")
    with pytest.raises(ValueError, match="dtype"):
        norm.forward(t["x"].float(), t["y"], **p)
    with pytest.raises(ValueError, match="elements"):
        norm.forward(t["x"][:3], t["y"], **p)
    with pytest.raises(ValueError, match="contiguous"):
        norm.forward(t["x"], torch.zeros((64, 4), dtype=torch.bfloat16, device=t["x"].device).t(), **p)
    with pytest.raises(ValueError, match="is on cpu"):
        norm.forward(t["x"].cpu(), t["y"], **p)
    with pytest.raises(ValueError, match="elements"):
        norm.forward(t["x"], t["y"], **dict(p, gate=p["gate"][:5]))
    with pytest.raises(B.OccultError):
        norm.forward(t["x"], t["y"], post_weight=p["post_weight"])      # its gate is missing
    with pytest.raises(ValueError):
        BlockNorm(4, 64, post="batch")
    with pytest.raises(B.OccultError):
        BlockNorm(4, 68)
    with pytest.raises(B.OccultError):
        BlockNorm(4, 64, pre_eps=0.0)


def test_replays_from_a_graph_and_on_another_stream():
    """Forward and backward captured once; every replay against the eager result, with eager work in between; two graphs of one
    object share its workspace, whose contents no call relies on."""
    norm, t, p, *_ = case(300, 2048, "bf16", "rms", "layer", "channel", seed=13)

    def step():
        out, h = norm.forward(t["x"], t["y"], **p)
        g = norm.backward(out, t["dout"], t["dh"], t["y"], **p)
        return [out, h] + [v for v in g.values() if v is not None]

    step()
    torch.cuda.synchronize()
    graphs = []
    side = torch.cuda.Stream()
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            res = step()
        graphs.append((graph, res))
        torch.cuda.synchronize()
    for rep in range(4):
        for n in ("x", "y", "dout", "dh"):
            t[n].copy_(torch.randn(t[n].shape, generator=torch.Generator().manual_seed(rep * 7 + len(n))).to(t[n].dtype))
        ref = [v.clone() for v in step()]
        graph, res = graphs[rep % 2]
        for v in res:
            v.fill_(3.0)
        norm.ws.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(res, ref)):
            assert torch.equal(a, b), (rep, i)
        with torch.cuda.stream(side):
            for i, (a, b) in enumerate(zip(step(), ref)):
                assert torch.equal(a, b), (rep, i, "side stream")
        torch.cuda.synchronize()
