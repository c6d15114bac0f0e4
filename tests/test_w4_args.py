"""4-bit expert weights on the host: the oracle's closed forms, and what the entry points refuse before any HIP call."""
import ctypes

import numpy as np
import pytest

from oracle import w4
from paper_2505_13345_amd import binding as B

P = 1 << 20          # an address that is never read
GOOD = dict(T=4, d=64, f=96, E=4, S=1, k=2, D=2, dtype="bf16")


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def weights(group=32, with_zeros=True, **change):
    q = B.occult_w4_weights_t(group)
    for i in range(3):
        q.codes[i], q.scales[i], q.zeros[i] = P, P, P if with_zeros else None
    for name, (i, v) in change.items():
        getattr(q, name)[i] = v
    return q


def test_oracle_rounds_to_nearest_and_packs():
    w = np.array([[7.0, -7.0, 3.4, 0.5, -0.5, 1.5, 0.0, -3.6]])
    codes, scales, zeros = w4.quantize(w, 32, False)
    assert scales.tolist() == [[1.0]] and zeros.tolist() == [[8]]
    assert codes.tolist() == [[15, 1, 11, 8, 8, 10, 8, 4]]           # ties to even
    assert w4.values(codes, scales, zeros, 32).tolist() == [[7.0, -7.0, 3.0, 0.0, 0.0, 2.0, 0.0, -4.0]]
    packed = w4.pack_bytes(codes)
    assert packed.tolist() == [[15 | 1 << 4, 11 | 8 << 4, 8 | 10 << 4, 8 | 4 << 4]]
    assert np.array_equal(w4.unpack_bytes(packed), codes)
    codes, scales, zeros = w4.quantize(np.array([[0.0, 15.0, -0.0, 7.2]]), 32, True)
    assert scales.tolist() == [[1.0]] and zeros.tolist() == [[0]] and codes.tolist() == [[0, 15, 0, 7]]
    codes, scales, zeros = w4.quantize(np.array([[-15.0, -1.0, -2.0, -3.0]]), 32, True)
    assert zeros.tolist() == [[15]] and codes.tolist() == [[0, 14, 13, 12]]
    codes, scales, zeros = w4.quantize(np.zeros((1, 4)), 32, True)
    assert scales.tolist() == [[0.0]] and codes.tolist() == [[8, 8, 8, 8]] and zeros.tolist() == [[8]]
    assert w4.bf16(np.array([1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8, 257.0])).tolist() == [1.0, 1.0 + 2.0 ** -6, 256.0]


def test_sizes(lib):
    cfg = B.make_cfg(**GOOD)
    n, kb = 5, 1                                    # experts; K blocks of 128 in 64 and in 96
    up = lambda v: (v + 255) // 256 * 256
    for group, zeros, per_scale in ((32, False, 2), (128, True, 4)):
        G = 128 // group
        pair, down = n * 6 * kb * 2, n * 4 * kb     # units of 16 rows: 96 / 16 in pairs, 64 / 16
        want = sum(up(b * 1024) + up(b * 16 * G * per_scale) for b in (pair, down))
        assert B.occult_pack_w4_bytes(cfg, group, zeros) == want


@pytest.mark.parametrize("kw,group,zeros,code", [
    (dict(), 16, 0, -1), (dict(), 96, 0, -1), (dict(), 0, 0, -1), (dict(), 32, 2, -1), (dict(d=68), 32, 0, -3), (dict(f=100), 32, 0, -3),
    (dict(dtype="f32", d=66), 32, 0, -3), (dict(E=5), 32, 0, -2)])
def test_layers_and_groups_refused(lib, kw, group, zeros, code):
    n = ctypes.c_size_t(0)
    cfg = B.make_cfg(**dict(GOOD, **kw))
    assert lib.occult_pack_w4_bytes(ctypes.byref(cfg), group, zeros, ctypes.byref(n)) == code
    assert lib.occult_expert_ffn_w4(ctypes.byref(cfg), None, P, P, P, 1 << 30, group, zeros, P, P, P, P, None) == code
    if group in (32, 64, 128) and zeros < 2:
        q = weights(group)
        assert lib.occult_pack_w4(ctypes.byref(cfg), ctypes.byref(q), P, 1 << 30, None) == code
        assert lib.occult_dequantize_weights(ctypes.byref(cfg), ctypes.byref(q), P, P, P, None) == code


@pytest.mark.parametrize("change,code", [
    (dict(codes=(1, None)), -4), (dict(scales=(2, None)), -4), (dict(zeros=(1, None)), -4), (dict(codes=(0, P + 4)), -3),
    (dict(scales=(0, P + 1)), -3)])
def test_weights_that_do_not_hold_together(lib, change, code):
    cfg, q = B.make_cfg(**GOOD), weights(**change)
    w = B.occult_weights_t(P, P, P)
    assert lib.occult_quantize_weights(ctypes.byref(cfg), ctypes.byref(w), ctypes.byref(q), None) == code
    assert lib.occult_dequantize_weights(ctypes.byref(cfg), ctypes.byref(q), P, P, P, None) == code
    assert lib.occult_pack_w4(ctypes.byref(cfg), ctypes.byref(q), P, 1 << 30, None) == code


def test_buffers(lib):
    cfg, q = B.make_cfg(**GOOD), weights()
    w = B.occult_weights_t(P, P, None)
    ref = ctypes.byref
    need = B.occult_pack_w4_bytes(cfg, 32, True)
    assert lib.occult_quantize_weights(ref(cfg), ref(w), ref(q), None) == -4
    assert lib.occult_quantize_weights(ref(cfg), ref(B.occult_weights_t(P, P + 8, P)), ref(q), None) == -3
    assert lib.occult_quantize_weights(ref(cfg), ref(w), None, None) == -4
    assert lib.occult_dequantize_weights(ref(cfg), ref(q), P, None, P, None) == -4
    assert lib.occult_dequantize_weights(ref(cfg), ref(q), P, P, P + 2, None) == -3
    assert lib.occult_pack_w4(ref(cfg), ref(q), None, need, None) == -4
    assert lib.occult_pack_w4(ref(cfg), ref(q), P + 8, need, None) == -3
    assert lib.occult_pack_w4(ref(cfg), ref(q), P, need - 1, None) == -5
    plan = B.occult_plan_t(*([P] * 12))
    call = lambda p=plan, sfd=P, x=P, packed=P, size=need, h=P, y=P, hs=P, ys=P: lib.occult_expert_ffn_w4(
        ref(cfg), ref(p) if p else None, sfd, x, packed, size, 32, 1, h, y, hs, ys, None)
    assert call(p=None) == -4 and call(p=B.occult_plan_t()) == -4
    for kw in (dict(sfd=None), dict(x=None), dict(packed=None), dict(h=None), dict(y=None), dict(hs=None), dict(ys=None)):
        assert call(**kw) == -4, kw
    for kw in (dict(sfd=P + 2), dict(x=P + 8), dict(packed=P + 4), dict(h=P + 2), dict(ys=P + 2)):
        assert call(**kw) == -3, kw
    assert call(size=need - 1) == -5
    buf = B.occult_forward_buffers_t()
    assert lib.occult_forward_w4(ref(cfg), ref(plan), None, P, P, need, 32, 1, None, None) == -4
    assert lib.occult_forward_w4(ref(cfg), ref(plan), None, P, P, need, 32, 1, ref(buf), None) == -4
    assert B.occult_last_error()
