"""A backward pass whose first call is the captured one: its sums over tokens start from zero once, not with every replay."""
import pytest
import torch

from tests.test_gpu_block_norm import case

pytestmark = pytest.mark.gpu

SUMS = ("dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias", "dgate")


def _captured(call):
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        res = call()
    torch.cuda.synchronize()
    return graph, res


def _eager(calls, **kw):
    norm, t, p, *_ = case(70, 264, "f32", "layer", "layer", "channel", seed=31)
    out, _ = norm.forward(t["x"], t["y"], **p)
    for accumulate in calls:
        g = norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=accumulate, **p)
    return {n: v.clone() for n, v in g.items()}


def test_replays_accumulate():
    norm, t, p, *_ = case(70, 264, "f32", "layer", "layer", "channel", seed=31)
    out, _ = norm.forward(t["x"], t["y"], **p)
    graph, g = _captured(lambda: norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=True, **p))
    for n in (1, 2, 3):
        want = _eager([True] * n)
        graph.replay()
        torch.cuda.synchronize()
        for name, v in want.items():
            assert torch.equal(g[name], v), (n, name)
    # and the same buffers go on with an eager call
    want = _eager([True] * 4)
    g = norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=True, **p)
    for name in SUMS:
        assert torch.equal(g[name], want[name]), name


def test_replay_then_an_accumulating_call():
    norm, t, p, *_ = case(70, 264, "f32", "layer", "layer", "channel", seed=31)
    out, _ = norm.forward(t["x"], t["y"], **p)
    graph, _ = _captured(lambda: norm.backward(out, t["dout"], t["dh"], t["y"], **p))
    for rep in range(2):
        graph.replay()
        torch.cuda.synchronize()
    g = norm.backward(out, t["dout"], t["dh"], t["y"], accumulate=True, **p)
    want = _eager([False, True])
    for name in SUMS:
        assert torch.equal(g[name], want[name]), name


@pytest.mark.parametrize("gate", ["token", "element"])
def test_gradients_per_token_from_a_captured_first_call(gate):
    norm, t, p, *_ = case(33, 520, "bf16", "rms", "rms", gate, seed=32)
    out, _ = norm.forward(t["x"], t["y"], **p)
    graph, g = _captured(lambda: norm.backward(out, t["dout"], t["dh"], t["y"], **p))
    other, *_ = case(33, 520, "bf16", "rms", "rms", gate, seed=32)
    want = {n: v.clone() for n, v in other.backward(out, t["dout"], t["dh"], t["y"], **p).items() if v is not None}
    for rep in range(3):
        for v in g.values():
            if v is not None:
                v.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, v in want.items():
            assert torch.equal(g[name], v), (rep, name)
