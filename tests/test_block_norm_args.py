"""What the block norm's entry points refuse, on the host: no kernel is launched here."""
import ctypes

import pytest

from paper_2505_13345_amd import binding as B

P = 1 << 20          # an address that is never read: every check comes before the first HIP call
RMS, LAYER = B.OCCULT_NORM_RMS, B.OCCULT_NORM_LAYER


@pytest.fixture(scope="module")
def lib():
    return B.load_library()


def desc(**kw):
    base = dict(post_kind=RMS, pre_kind=RMS, gate_kind=0, x_scale=1.0, y_scale=1.0, post_eps=1e-6, pre_eps=1e-6, weight_offset=0.0)
    return B.occult_block_norm_t(**dict(base, **kw))


def cfg(T=4, d=64, dtype="bf16"):
    return B.make_cfg(T, d, d, 1, 0, 1, 1, dtype)


def forward(lib, n, c=None, x=P, y=2 * P, out=3 * P, h=4 * P):
    return lib.occult_block_norm(ctypes.byref(c or cfg()), ctypes.byref(n), x, y, out, h, None)


def backward(lib, n, c=None, y=P, out=2 * P, dout=3 * P, dh=4 * P, dx=5 * P, dy=6 * P, grads=None, accumulate=0, ws=None, ws_bytes=0):
    g = grads or B.occult_block_norm_grads_t()
    return lib.occult_block_norm_backward(ctypes.byref(c or cfg()), ctypes.byref(n), y, out, dout, dh, dx, dy, ctypes.byref(g),
                                          accumulate, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,code", [
    (dict(post_kind=3), -1), (dict(pre_kind=-1), -1), (dict(gate_kind=4, gate=P), -1),
    (dict(x_scale=float("nan")), -1), (dict(y_scale=float("inf")), -1), (dict(weight_offset=float("nan")), -1),
    (dict(post_eps=0.0), -1), (dict(pre_eps=-1e-6), -1), (dict(pre_eps=float("inf")), -1),
    (dict(post_kind=0, post_weight=P), -1), (dict(pre_kind=0, pre_bias=P), -1),
    (dict(gate_kind=1), -4), (dict(gate=P), -4),
    (dict(post_weight=P + 8), -3), (dict(gate_kind=3, gate=P + 2), -3), (dict(gate_kind=2, gate=P + 1), -3)])
def test_descriptions_that_do_not_hold_together(lib, kw, code):
    assert forward(lib, desc(**kw)) == code
    assert backward(lib, desc(**kw)) == code
    n = ctypes.c_size_t(0)
    assert lib.occult_block_norm_backward_ws_bytes(ctypes.byref(cfg()), ctypes.byref(desc(**kw)), ctypes.byref(n)) == code
    assert B.occult_last_error()


def test_shapes(lib):
    assert forward(lib, desc(), cfg(d=68)) == -3                       # rows of 136 bytes
    assert forward(lib, desc(), cfg(d=16392)) == -2                    # rows beyond 32768 bytes
    assert forward(lib, desc(), cfg(d=8196, dtype="f32")) == -2
    assert lib.occult_block_norm(None, ctypes.byref(desc()), P, P, P, P, None) == -4
    assert lib.occult_block_norm(ctypes.byref(cfg()), None, P, P, P, P, None) == -4


@pytest.mark.parametrize("kw,args,code", [
    ({}, dict(x=None), -4), ({}, dict(out=None), -4), ({}, dict(h=None), -4), ({}, dict(x=P + 2), -3), ({}, dict(h=3 * P), -1),
    ({}, dict(y=None), -1),                                            # a post norm of nothing
    (dict(post_kind=0, gate_kind=2, gate=P), dict(y=None), -1), (dict(post_kind=0, pre_kind=0), dict(y=None), -1)])
def test_forward_buffers(lib, kw, args, code):
    assert forward(lib, desc(**kw), **args) == code


@pytest.mark.parametrize("kw,args,code", [
    ({}, dict(out=None), -4), ({}, dict(dh=None), -4), ({}, dict(y=None), -4), ({}, dict(dx=None, dy=None), -4),
    (dict(pre_kind=0), dict(dout=None), -4), ({}, dict(dx=6 * P), -1), ({}, dict(dy=6 * P + 4), -3), ({}, dict(accumulate=2), -1),
    ({}, dict(grads=B.occult_block_norm_grads_t(post_weight=P)), -1),  # of a weight that is not there
    (dict(post_weight=P), dict(grads=B.occult_block_norm_grads_t(post_weight=P), dy=None), -4),
    (dict(post_weight=P), dict(grads=B.occult_block_norm_grads_t(post_weight=P)), -5),
    (dict(post_weight=P), dict(grads=B.occult_block_norm_grads_t(post_weight=P), ws=P, ws_bytes=64 * 4 - 1), -5)])
def test_backward_buffers(lib, kw, args, code):
    assert backward(lib, desc(**kw), **args) == code


def test_workspace_counts_the_parameters(lib):
    one = B.occult_block_norm_backward_ws_bytes(cfg(), desc(post_weight=P))
    assert one >= 64 * 4
    assert B.occult_block_norm_backward_ws_bytes(cfg(), desc()) == 0
    assert B.occult_block_norm_backward_ws_bytes(cfg(), desc(post_weight=P, post_bias=P, pre_weight=P, pre_bias=P, gate_kind=1,
                                                             gate=P)) == 5 * one
    assert B.occult_block_norm_backward_ws_bytes(cfg(T=0), desc(post_weight=P)) == 0
    with pytest.raises(B.OccultError):
        B.occult_block_norm_backward_ws_bytes(cfg(d=68), desc())


def test_nothing_to_do_without_tokens(lib):
    assert forward(lib, desc(), cfg(T=0), None, None, None, None) == 0
    assert backward(lib, desc(), cfg(T=0), None, None, None, None, None, None) == 0
