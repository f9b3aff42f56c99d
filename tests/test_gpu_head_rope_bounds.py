"""Norm and rotation of heads on the GPU: channels that are passed through."""
import numpy as np
import pytest

from attention_util import rope_graph, rope_reference
from test_gpu_attention import MODES, run
from paper_2012_02732_amd import binding as B
from workloads import rope_frequencies

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("tokens", [1, 5, 16, 70])
@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("d,rot", [(16, 8), (9, 2), (150, 100)])
def test_infinities_in_channels_that_are_not_rotated_stay_there(tokens, interleaved, d, rot):
    """A channel behind the rotated ones is passed as it is: what it holds reaches no other channel, forward or backward."""
    rng = np.random.default_rng(tokens + d)
    x, dy = (rng.standard_normal((2, 2 * d, 1, tokens)).astype(np.float32) for _ in range(2))
    bad = [rot, d - 1]                                          # the first of them, which has a neighbour, and the last
    pos = rng.integers(0, 1000, (2, 1, 1, tokens)).astype(np.float32)
    clean = rope_reference(x, pos, rope_frequencies(rot), None, dy, 2, interleaved, 0.0, 1.0)
    for value in (np.inf, -np.inf, np.nan):
        xb, yb = x.copy(), dy.copy()
        for c in bad:
            xb[0, c, 0, 0], xb[1, d + c, 0, -1] = value, value
            yb[0, c, 0, 0], yb[1, d + c, 0, -1] = value, value
        got = run(rope_graph(xb, pos, rope_frequencies(rot), None, yb, 2, interleaved, 0.0, 1.0), MODES)
        for mode, tensors in got.items():
            for name, like in (("y", xb), ("dx", yb)):
                t = tensors[name]
                hit = ~np.isfinite(like)
                assert np.array_equal(t[hit], like[hit], equal_nan=True), (mode, name, value)
                assert np.isfinite(t[~hit]).all(), (mode, name, value)
                off = np.abs(t - clean[name])[~hit].max()
                assert off <= 8 * U * np.abs(clean[name]).max(), (mode, name, off)


@pytest.mark.parametrize("tokens", [5, 16, 70])
def test_gradient_of_gamma_next_to_infinities(tokens):
    """dgamma of a channel that is passed through comes from this channel alone."""
    rng = np.random.default_rng(tokens)
    x, dy = (rng.standard_normal((2, 32, 1, tokens)).astype(np.float32) for _ in range(2))
    pos, gamma = np.zeros((1, 1, 1, tokens), np.float32), np.ones(16, np.float32)
    clean = rope_reference(x, pos, rope_frequencies(8), gamma, dy, 2, 0, 1e-6, 1.0)["dgamma"]
    dy[1, 16 + 9, 0, 3] = np.inf
    got = run(rope_graph(x, pos, rope_frequencies(8), gamma, dy, 2, 0, 1e-6, 1.0))[B.NG_MODE_GRAPH_SINGLE]["dgamma"]
    assert np.isinf(got[0, 9, 0, 0])
    others = [c for c in range(16) if c != 9]
    # a sum of 4 tokens terms of order one
    assert np.abs(got - clean)[0, others].max() <= 4 * U * 4 * tokens
