"""The oracle's gradients of the pre norm alone, h = N_pre(x), against differences of its own forward pass."""
import numpy as np
import pytest

from oracle import block_norm as bn


@pytest.mark.parametrize("pre", ["rms", "layer"])
@pytest.mark.parametrize("stream", [False, True])
def test_gradients_of_the_pre_norm_alone_equal_differences(pre, stream):
    """A step of 1e-5 leaves about 1e-10 from the third derivative and 1e-11 from rounding, relative to values of a few tens.
    stream: x is also read beside h, with a gradient of its own."""
    rng = np.random.default_rng(4)
    T, d = 3, 5
    cfg = dict(post=None, pre=pre, gate=None, x_scale=0.5, y_scale=-1.3, offset=1.0, post_eps=0.1, pre_eps=0.2)
    p = {"pre_weight": rng.standard_normal(d), "pre_bias": rng.standard_normal(d)}
    x, dout, dh = (rng.standard_normal((T, d)) for _ in range(3))

    def loss():
        return (dh * bn.pre_norm(x, cfg, p)[0]).sum() + ((dout * x).sum() if stream else 0.0)

    got = bn.gradients(x, None, dout if stream else None, dh, cfg, p)
    leaves = dict({"d" + n: t for n, t in p.items()}, dx=x)
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
