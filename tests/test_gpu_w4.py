"""4-bit expert weights against the float64 oracle: rounding and packing exactly, the expert network step by step.

Bars of the network.  A group's sum of 32 to 128 products (16 + code) * x, and of -(16 + zero) * x, passes at most 2 * 128 roundings of
2^-24 of a partial sum of at most 31 * sum |x|: 2^-16 * 31 * scale * sum |x| for its part of a result; the sums of the groups add
(K / 32 + 4) * 2^-24 <= 2^-17 of the sum of their magnitudes, and SwiGLU a few units in the last place (2^-20 of h).  h is
compared with x, and y with the h that the GPU stored, so each carries one rounding to the storage type.  The mean error is bounded
far below that worst case: the roundings are independent, so their sum grows with the root of their number, sqrt(256) * 2^-25 *
24 * sqrt(K) |x| scale against results of 2.7 * sqrt(K) |x| scale: 5e-6 of the result's rms; bar 2e-5, beside half a step of the
storage type."""
import numpy as np
import pytest
import torch

from inputs import workloads as wl
from oracle import block_norm as bn
from oracle import moe_std, w4
from paper_2505_13345_amd import binding as B
from paper_2505_13345_amd.layer import OccultLayer, W4Weights
from paper_2505_13345_amd.norm import BlockNorm
from tests.helpers import BF16_U, require_gpu, say

pytestmark = pytest.mark.gpu

MATS = ("gate", "up", "down")


def make(T, d, f, E, S, k, D, dtype, group, zeros, seed=0, placement=None, spread=1.0):
    """A layer with random 4-bit weights, packed, and a routed batch: layer, x on the GPU, oracle weights (value, scale * 31)."""
    dev = require_gpu()
    rng = np.random.default_rng(seed)
    pos = None if placement is None else wl.random_placement(E, D, seed=placement)
    layer = OccultLayer(T, d, f, E, S, k, D, dtype, expert_pos=pos)
    x = (rng.standard_normal((T, d)) * spread).astype(np.float32)
    if dtype == "bf16":
        x = wl.round_to_bf16(x)
    codes, scales, zps, values, tops = [], [], [], [], []
    for rows, K in ((f, d), (f, d), (d, f)):
        groups = (K + group - 1) // group
        q = np.clip(np.rint(rng.standard_normal((E + S, rows, K)) * 2.7) + 8, 0, 15).astype(np.int64)
        s = w4.bf16(rng.uniform(0.7, 1.4, (E + S, rows, groups)) / (2.7 * np.sqrt(K)))
        z = rng.integers(0, 16, (E + S, rows, groups)) if zeros else np.full((E + S, rows, groups), 8)
        to = lambda a, dt: torch.from_numpy(np.ascontiguousarray(a)).to(dev).to(dt)
        codes.append(to(w4.pack_bytes(q), torch.uint8))
        scales.append(to(s, torch.bfloat16))
        zps.append(to(z.astype(np.uint8), torch.uint8) if zeros else None)
        values.append(w4.values(q, s, z, group))
        tops.append(31.0 * s[..., np.arange(K) // group])
    weights = W4Weights(group, tuple(codes), tuple(scales), tuple(zps) if zeros else None)
    layer.pack_weights_w4(weights)
    logits = torch.from_numpy(rng.standard_normal((T, E)).astype(np.float32)).to(dev)
    xd = torch.from_numpy(x).to(dev).to(layer.tdtype)
    layer.route(logits)
    layer.make_plan()
    layer.dispatch(xd)
    return layer, xd, logits, weights, values, tops, x.astype(np.float64)


def f64(t):
    return t.detach().cpu().double().numpy()


def compare(got, want, terms, tops, dtype, what):
    """terms: sums of the magnitudes of the products, tops: of 31 * scale * |x|."""
    u = BF16_U if dtype == "bf16" else 2.0 ** -24
    err = np.abs(got - want)
    bar = u * (1 + 2.0 ** -7) * np.abs(want) + 2.0 ** -16 * tops + 2.0 ** -17 * terms + 2.0 ** -20 * np.abs(want)
    assert np.isfinite(got).all() and (err <= bar).all(), f"{what}: {(err - bar).max():.3e} beyond the bar"
    rms = np.sqrt(np.mean(want ** 2))
    assert err.mean() <= (u / 2 + 2e-5) * rms, f"{what}: mean error {err.mean() / rms:.2e} of the rms"


def check_network(layer, x, values, tops, dtype, what):
    s = layer.shape
    E, S, f = s["E"], s["S"], s["f"]
    tabs = {n: v.cpu().numpy() for n, v in layer.tables().items()}
    h_all, y_all = f64(layer.epd_h), f64(layer.epd_y)
    src = tabs["sfd_token"][tabs["epd_sfd_row"]]

    def one(e, rows, h, y, y_of, what):
        g, up = rows @ values[0][e].T, rows @ values[1][e].T
        silu = g / (1.0 + np.exp(-g))
        a = np.abs(rows)
        mag = lambda m: (a @ np.abs(values[m][e]).T, a @ tops[m][e].T)
        (tg, pg), (tu, pu) = mag(0), mag(1)
        # |silu'| <= 1.1, |silu(g)| <= |g|
        compare(h, silu * up, 1.1 * tg * np.abs(up) + np.abs(g) * tu + 1.1 * np.abs(g) * np.abs(up), 1.1 * pg * np.abs(up) + np.abs(g) * pu,
                dtype, what + " h")
        y_of.append((h @ values[2][e].T, np.abs(h) @ np.abs(values[2][e]).T, np.abs(h) @ tops[2][e].T))

    for p in range(E):
        lo, hi = tabs["exp_offset"][p], tabs["exp_offset"][p + 1]
        if lo == hi:
            continue
        res = []
        one(tabs["pos_expert"][p], x[src[lo:hi]], h_all[lo:hi], None, res, f"{what} expert at {p}")
        compare(y_all[lo:hi], *res[0], dtype, f"{what} expert at {p} y")
    if S:
        hs, res = f64(layer.h_shared), []
        for i in range(S):
            one(E + i, x, hs[:, i * f:(i + 1) * f], None, res, f"{what} shared {i}")
        compare(f64(layer.y_shared), *(sum(r[n] for r in res) for n in range(3)), dtype, f"{what} shared y")


# (T, d, f, E, S, k, D): one token; K and N below, at and beyond a code block; shared experts; odd widths; experts without rows; more
# rows per expert than a tile; a single expert for all
SHAPES = [(1, 64, 64, 4, 0, 1, 1), (1, 136, 72, 8, 1, 2, 2), (2, 128, 128, 4, 2, 4, 2), (17, 264, 200, 6, 0, 3, 3), (33, 256, 384, 8, 3, 2, 4),
          (64, 520, 136, 16, 0, 4, 4), (150, 128, 256, 2, 1, 1, 1), (200, 72, 40, 1, 0, 1, 1), (5, 1024, 512, 64, 2, 6, 16), (300, 96, 160, 4, 2, 2, 2)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, False), (32, True), (64, False), (128, True)])
def test_network(shape, group, zeros):
    say(f"{shape} group {group} zeros {zeros}")
    layer, xd, _, _, values, tops, x = make(*shape, "bf16", group, zeros, seed=sum(shape))
    for t in (layer.epd_h, layer.epd_y):
        t.fill_(7.0)
    epd_y, y_shared = layer.expert_ffn_w4(xd)
    assert epd_y is layer.epd_y and y_shared is layer.y_shared
    check_network(layer, x, values, tops, "bf16", f"{shape} {group} {zeros}")


@pytest.mark.parametrize("shape", [(1, 64, 64, 4, 0, 1, 1), (9, 68, 36, 4, 1, 2, 2), (40, 132, 260, 8, 2, 2, 4), (256, 128, 256, 16, 0, 4, 4)])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, True), (128, False)])
def test_network_f32(shape, group, zeros):
    say(f"f32 {shape} group {group} zeros {zeros}")
    layer, xd, _, _, values, tops, x = make(*shape, "f32", group, zeros, seed=sum(shape))
    layer.expert_ffn_w4(xd)
    check_network(layer, x, values, tops, "f32", f"f32 {shape} {group} {zeros}")


# enough workgroups for the kernels whose waves take the whole K (the layers above are computed with K split over the waves): 16-row tiles
# in the first and in the second product; shared experts' long sums split, and with codes three blocks ahead; 32-row tiles, with
# one and with two units per wave; odd widths, experts without rows, tiles with one and two blocks of rows
TILED = [(20, 200, 648, 64, 4, 4, 4), (20, 648, 200, 64, 4, 4, 4), (18, 648, 640, 64, 4, 4, 4), (50, 648, 1032, 64, 4, 2, 4),
         (70, 648, 1032, 64, 4, 3, 4), (60, 72, 1416, 16, 1, 4, 4), (60, 1416, 72, 16, 0, 4, 4), (60, 136, 2008, 8, 1, 4, 2),
         (60, 2008, 136, 8, 0, 4, 2), (130, 264, 1928, 4, 2, 2, 2), (130, 1928, 264, 4, 2, 2, 2)]


@pytest.mark.parametrize("shape", TILED)
@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, False), (64, True), (128, False), (128, True)])
def test_network_in_tiles(shape, group, zeros):
    say(f"tiles {shape} group {group} zeros {zeros}")
    layer, xd, _, _, values, tops, x = make(*shape, "bf16", group, zeros, seed=sum(shape))
    layer.expert_ffn_w4(xd)
    check_network(layer, x, values, tops, "bf16", f"{shape} {group} {zeros}")
    first = [t.clone() for t in (layer.epd_y, layer.epd_h) + ((layer.y_shared, layer.h_shared) if shape[4] else ())]
    layer.expert_ffn_w4(xd)
    for a, b in zip(first, (layer.epd_y, layer.epd_h) + ((layer.y_shared, layer.h_shared) if shape[4] else ())):
        assert torch.equal(a, b)   # sums in a fixed order


def test_placed_experts_and_a_large_batch():
    layer, xd, _, _, values, tops, x = make(2500, 136, 72, 8, 1, 3, 4, "bf16", 64, True, seed=3, placement=5)
    layer.expert_ffn_w4(xd)
    check_network(layer, x, values, tops, "bf16", "placed")


def test_rows_beyond_4_gib():
    """x, sfd_x, epd_y and y_shared of 4.5 GB: rows at both ends and around the border against the oracle."""
    dev = require_gpu()
    T, d, f, E, S, k = 550_000, 4096, 64, 4, 1, 1
    small = make(8, d, f, E, S, k, 1, "bf16", 128, True, seed=13)
    values, tops = small[4], small[5]
    layer = OccultLayer(T, d, f, E, S, k, 1)
    layer.pack_weights_w4(small[3])
    gen = torch.Generator(device=dev).manual_seed(5)
    xd = torch.randn((T, d), device=dev, generator=gen, dtype=torch.bfloat16)
    layer.route(torch.randn((T, E), device=dev, generator=gen))
    layer.make_plan()
    layer.dispatch(xd)
    layer.expert_ffn_w4(xd)
    offset = layer.tables()["exp_offset"].cpu().numpy()
    src = layer.tables()["sfd_token"][layer.tables()["epd_sfd_row"].long()]
    for row in (0, 1, 524_287, 524_288, T - 1):
        e, t = int(np.searchsorted(offset, row, side="right") - 1), int(src[row])
        for expert, rows, h, y in ((e, t, layer.epd_h[row], layer.epd_y[row]), (E, row, layer.h_shared[row], layer.y_shared[row])):
            x = f64(xd[rows])
            g, up = values[0][expert] @ x, values[1][expert] @ x
            want = g / (1.0 + np.exp(-g)) * up
            h = f64(h)
            assert np.abs(h - want).max() <= 2 * BF16_U * np.abs(want).max(), (row, "h")
            compare(f64(y), values[2][expert] @ h, np.abs(values[2][expert]) @ np.abs(h), tops[2][expert] @ np.abs(h), "bf16", f"row {row} y")


def test_phases_and_rows_behind_the_last():
    """The two products one by one give the same bits; scratch rows behind the batch's stay as they were."""
    dev = require_gpu()
    layer, xd, _, _, *_ = make(7, 264, 200, 6, 1, 3, 3, "bf16", 32, False, seed=4)
    ref = [t.clone() for t in (layer.expert_ffn_w4(xd)[0], layer.y_shared, layer.epd_h, layer.h_shared)]
    pad = [torch.full((t.shape[0] + 3, t.shape[1]), 7.0, dtype=t.dtype, device=dev) for t in ref]
    for phase in (1, 2):
        layer.cfg.ffn_phase = phase
        B.occult_expert_ffn_w4(layer.cfg, layer.plan, layer.sfd_x, xd, *layer._packed_w4(), pad[2], pad[0], pad[3], pad[1])
        if phase == 1:
            assert (pad[0] == 7.0).all() and (pad[1] == 7.0).all()
    layer.cfg.ffn_phase = 0
    for p, r in zip(pad, ref):
        assert torch.equal(p[:r.shape[0]], r) and (p[r.shape[0]:] == 7.0).all()


def test_infinities_and_nan_stay_in_their_rows():
    layer, xd, _, _, *_ = make(40, 136, 72, 4, 1, 2, 2, "bf16", 32, True, seed=6)
    ref = [t.clone() for t in layer.expert_ffn_w4(xd)]
    src = layer.tables()["sfd_token"][layer.tables()["epd_sfd_row"].long()]
    xd[3, 5], xd[11, 7] = float("inf"), float("nan")
    layer.dispatch(xd)
    got = layer.expert_ffn_w4(xd)
    bad = (src == 3) | (src == 11)
    assert torch.equal(got[0][~bad], ref[0][~bad]) and not torch.isfinite(got[0][bad]).all(dim=1).any()
    keep = [i for i in range(40) if i not in (3, 11)]
    assert torch.equal(got[1][keep], ref[1][keep])


@pytest.mark.parametrize("dtype,d,f", [("bf16", 136, 72), ("bf16", 256, 128), ("f32", 68, 100)])
@pytest.mark.parametrize("group,zeros", [(32, False), (64, True), (128, True)])
def test_quantised_weights_equal_the_oracle(dtype, d, f, group, zeros):
    dev = require_gpu()
    rng = np.random.default_rng(d + group)
    layer = OccultLayer(1, d, f, 3, 1, 1, 1, dtype)
    w = [rng.standard_normal((4, *s)).astype(np.float32) * 0.02 for s in ((f, d), (f, d), (d, f))]
    for a in w:
        a[0, 0, :] = 0.0                                    # groups of zeros
        a[0, 1, :40] = np.abs(a[0, 1, :40])                 # one sign
        a[0, 2, :40] = -np.abs(a[0, 2, :40])
        a[0, 3, :] = np.rint(a[0, 3, :] * 200) / 2.0        # multiples of 1/2: quotients on rounding borders
        a[0, 3, 0] = 7.0
        a[0, 4, :] *= 1e-30
        a[0, 5, :] *= 1e30
    if dtype == "bf16":
        w = [wl.round_to_bf16(a) for a in w]
    wd = [torch.from_numpy(a).to(dev).to(layer.tdtype) for a in w]
    q = layer.quantize_weights(*wd, group=group, zeros=zeros)
    back = layer.dequantize_weights(q)
    for i, name in enumerate(MATS):
        codes, scales, zps = w4.quantize(w[i].astype(np.float64), group, zeros)
        assert np.array_equal(q.codes[i].cpu().numpy(), w4.pack_bytes(codes)), name
        assert np.array_equal(f64(q.scales[i]), scales), name
        if zeros:
            assert np.array_equal(q.zeros[i].cpu().numpy(), zps), name
        want = w4.values(codes, scales, zps, group)
        want = w4.bf16(want) if dtype == "bf16" else want.astype(np.float32).astype(np.float64)
        assert np.array_equal(f64(back[i]), want), name


def test_forward_in_one_call_and_step_by_step():
    layer, xd, logits, q, values, *_ = make(24, 128, 192, 8, 2, 3, 4, "bf16", 64, False, seed=8)
    y = layer.forward_w4(logits, xd).clone()
    layer.route(logits)
    layer.make_plan()
    layer.dispatch(xd)
    layer.expert_ffn_w4(xd)
    layer.combine()
    assert torch.equal(layer.y, y)
    # the whole layer against the textbook layer on the same values: the bars of the bf16 layer
    ids, w = layer.ids.cpu().numpy(), f64(layer.w)
    ref = moe_std.moe_layer(f64(xd), ids, w, *(v.astype(np.float64) for v in values), 8, 2)
    rms = np.sqrt(np.mean(ref ** 2))
    # h, epd_y, sfd_y, y_shared and y are stored in bf16: five roundings, each of at most BF16_U of a value not larger than the rms in the mean
    assert np.abs(f64(y) - ref).mean() <= 5 * BF16_U / np.sqrt(3.0) * rms
    # and against the ordinary path on the values that the codes stand for, which are rounded once more there
    dense = layer.forward(logits, xd, *layer.dequantize_weights(q))
    assert np.abs(f64(dense) - ref).mean() <= 8 * BF16_U / np.sqrt(3.0) * rms


def test_own_steps_are_called():
    layer, xd, logits, *_ = make(5, 64, 64, 4, 0, 2, 2, "bf16", 32, False)
    seen = []
    combine = layer.combine
    layer.combine = lambda: (seen.append(1), combine())
    y = layer.forward_w4(logits, xd).clone()
    del layer.combine
    assert seen == [1] and torch.equal(layer.forward_w4(logits, xd), y)


def test_refusals_of_the_buffers():
    layer, xd, logits, q, *_ = make(5, 64, 96, 4, 0, 2, 2, "bf16", 32, True)
    with pytest.raises(ValueError, match="dtype"):
        layer.pack_weights_w4(q._replace(scales=tuple(s.float() for s in q.scales)))
    with pytest.raises(ValueError, match="elements"):
        layer.pack_weights_w4(q._replace(group=32, codes=tuple(c[:3] for c in q.codes)))
    with pytest.raises(B.OccultError):
        layer.pack_weights_w4(q._replace(group=48))
    with pytest.raises(ValueError, match="elements"):
        layer.expert_ffn_w4(xd[:2])
    with pytest.raises(ValueError, match="no 4-bit weights"):
        OccultLayer(5, 64, 96, 4, 0, 2, 2).expert_ffn_w4(xd)
    with pytest.raises(B.OccultError):
        layer.quantize_weights(*layer.dequantize_weights(q), group=20)
    with pytest.raises(ValueError, match="not in GPU memory"):
        layer.expert_ffn_w4(xd.cpu())


def test_refusal_of_another_current_device(monkeypatch):
    layer, xd, logits, *_ = make(5, 64, 96, 4, 0, 2, 2, "bf16", 32, True)
    norm = BlockNorm(5, 64)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: layer.expert_ffn_w4(xd), lambda: layer.forward_w4(logits, xd), lambda: norm.forward(xd),
                 lambda: norm.backward(xd, None, xd)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_weights_packed_again():
    """The same format goes to the same buffer, which a captured graph goes on reading; another format takes a new one."""
    layer, xd, _, q, *_ = make(9, 136, 72, 4, 1, 2, 2, "bf16", 32, True, seed=11)
    other = make(9, 136, 72, 4, 1, 2, 2, "bf16", 32, True, seed=12)[3]
    first = layer.expert_ffn_w4(xd)[0].clone()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        layer.expert_ffn_w4(xd)
    torch.cuda.synchronize()
    at = layer.packed_w4.data_ptr()
    layer.pack_weights_w4(other)
    assert layer.packed_w4.data_ptr() == at
    second = layer.expert_ffn_w4(xd)[0].clone()
    assert not torch.equal(first, second)
    for weights, want in ((q, first), (other, second), (q, first)):
        layer.pack_weights_w4(weights)
        layer.epd_y.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.epd_y, want)
    keep = layer.packed_w4
    layer.pack_weights_w4(layer.quantize_weights(*layer.dequantize_weights(q), group=64))
    assert layer.packed_w4.data_ptr() != keep.data_ptr()
    with pytest.raises(B.OccultError):
        layer.pack_weights_w4(q._replace(group=16))
    assert layer.w4_format == (64, False)


def test_no_tokens():
    layer, *_ = make(0, 64, 96, 4, 1, 2, 2, "bf16", 32, False)
    epd_y, y_shared = layer.expert_ffn_w4(torch.zeros((0, 64), dtype=torch.bfloat16, device=layer.device))
    assert epd_y.shape == (0, 64) and y_shared.shape == (0, 64)


def test_block_from_norm_to_norm():
    """A decode step of a block on the residual stream: pre norm, router, 4-bit experts, combine, post norm, gate, residual sum, next
    pre norm; each part against the oracle on what the part before it stored; captured once and replayed on changed inputs."""
    dev = require_gpu()
    T, d, f, E, S, k, D = 24, 256, 192, 8, 1, 2, 4
    layer, xd, _, q, values, tops, _ = make(T, d, f, E, S, k, D, "bf16", 64, True, seed=9)
    bf = lambda *s: torch.randn(s, device=dev, generator=gen).to(torch.bfloat16)
    gen = torch.Generator(device=dev).manual_seed(1)
    w_router, pre_w, post_w, next_w, gate = bf(E, d) * 0.06, bf(d), bf(d), bf(d), bf(d)
    first = BlockNorm(T, d, pre="rms", pre_eps=1e-5)
    norm = BlockNorm(T, d, post="rms", pre="rms", gate="channel", x_scale=1.0, y_scale=0.5)
    params = dict(gate=gate, post_weight=post_w, pre_weight=next_w)

    def step():
        _, h = first.forward(xd, pre_weight=pre_w)
        return layer.forward_block(xd, h, w_router, norm, **params)

    def check():
        p64 = {n: f64(v) for n, v in params.items()}
        cfg = dict(post="rms", pre="rms", gate="channel", x_scale=1.0, y_scale=0.5, post_eps=1e-6, pre_eps=1e-6, offset=0.0)
        h64 = f64(first.h)
        logits = f64(layer.logits)
        want = h64 @ f64(w_router).T
        assert np.abs(logits - want).max() <= 2.0 ** -17 * (np.abs(h64) @ np.abs(f64(w_router)).T).max()
        check_network(layer, h64, values, tops, "bf16", "block")
        ids, w = layer.ids.cpu().numpy(), f64(layer.w)
        ref = moe_std.moe_layer(h64, ids, w, *values, E, S)
        assert np.abs(f64(layer.y) - ref).mean() <= 5 * BF16_U / np.sqrt(3.0) * np.sqrt(np.mean(ref ** 2))
        value, scale = bn.stream(f64(xd), f64(layer.y), cfg, p64)
        assert (np.abs(f64(norm.out) - value) <= BF16_U * 1.01 * np.abs(value) + 2.0 ** -18 * scale).all()
        value, scale = bn.pre_norm(f64(norm.out), cfg, p64)
        assert (np.abs(f64(norm.h) - value) <= BF16_U * 1.01 * np.abs(value) + 2.0 ** -18 * scale).all()

    step()
    torch.cuda.synchronize()
    check()
    # the same block from the values in bf16 (the ordinary expert products)
    out = norm.out.clone()
    layer.forward_block(xd, first.h, w_router, norm, layer.dequantize_weights(q), **params)
    assert (out.float() - norm.out.float()).abs().mean() <= 0.02 * out.float().abs().mean()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    torch.cuda.synchronize()
    for rep in range(3):
        xd.copy_(bf(T, d) * (1 + rep))
        step()
        torch.cuda.synchronize()
        ref = [t.clone() for t in (norm.out, norm.h, layer.y, layer.ids, layer.epd_y)]
        for t in (norm.out, norm.h, layer.y, layer.epd_h, layer.epd_y, layer.h_shared):
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((norm.out, norm.h, layer.y, layer.ids, layer.epd_y), ref):
            assert torch.equal(a, b), rep
        check()
