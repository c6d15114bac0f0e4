"""The block norm's oracle: closed forms, and its gradients against differences of its own forward pass."""
import numpy as np
import pytest

from oracle import block_norm as bn

BASE = dict(post="rms", pre="rms", gate=None, x_scale=1.0, y_scale=1.0, post_eps=1e-6, pre_eps=1e-5, offset=0.0)


def test_closed_forms():
    v = np.array([[3.0, -4.0]])
    got, _ = bn.norm(v, "rms", 0.0)
    assert np.allclose(got, v / np.sqrt(12.5), rtol=1e-15)
    got, _ = bn.norm(v, "layer", 0.0, w=np.array([2.0, 2.0]), b=np.array([1.0, 1.0]), offset=1.0)
    assert np.allclose(got, [[4.0, -2.0]], rtol=1e-15)         # (v - mean) / std = +-1, times 3, plus 1
    assert np.allclose(bn.norm(np.zeros((1, 4)), "rms", 1e-6)[0], 0.0)
    out, _ = bn.stream(v, v, dict(BASE, post=None, x_scale=0.5, y_scale=2.0, gate="token"), dict(gate=np.array([3.0])))
    assert np.allclose(out, 6.5 * v, rtol=1e-15)


@pytest.mark.parametrize("post", [None, "rms", "layer"])
@pytest.mark.parametrize("pre", [None, "rms", "layer"])
@pytest.mark.parametrize("gate", [None, "channel", "token", "element"])
def test_gradients_equal_differences(post, pre, gate):
    """<dout, out> + <dh, h> by central differences in float64: a step of 1e-5 leaves an error of about 1e-10 from the
    third derivative and 1e-11 from rounding, relative to values of a few tens."""
    rng = np.random.default_rng(3)
    T, d = 3, 5
    cfg = dict(BASE, post=post, pre=pre, gate=gate, x_scale=0.7, y_scale=-1.3, offset=1.0, post_eps=0.1, pre_eps=0.2)
    p = {}
    for side, kind in (("post", post), ("pre", pre)):
        if kind:
            p[side + "_weight"] = rng.standard_normal(d)
            p[side + "_bias"] = rng.standard_normal(d)
    if gate:
        p["gate"] = rng.standard_normal({"channel": d, "token": T, "element": (T, d)}[gate])
    x, y, dout, dh = (rng.standard_normal((T, d)) for _ in range(4))

    def loss():
        out, _ = bn.stream(x, y, cfg, p)
        return (dout * out).sum() + ((dh * bn.pre_norm(out, cfg, p)[0]).sum() if pre else 0.0)

    got = bn.gradients(bn.stream(x, y, cfg, p)[0], y, dout, dh if pre else None, cfg, p)
    leaves = dict({"d" + n: t for n, t in p.items()}, dx=x, dy=y)
    assert set(got) == set(leaves)
    for name, leaf in leaves.items():
        flat = leaf.reshape(-1)
        for i in range(flat.size):
            keep = flat[i]
            flat[i] = keep + 1e-5
            up = loss()
            flat[i] = keep - 1e-5
            down = loss()
            flat[i] = keep
            assert abs((up - down) / 2e-5 - got[name][0].reshape(-1)[i]) <= 1e-7, name
