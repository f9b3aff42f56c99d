"""Norm and rotation of heads on the GPU: channels that are passed through, and angles of far positions."""
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


@pytest.mark.parametrize("tokens", [4, 64])
@pytest.mark.parametrize("base", [1e3, 2.0 ** 24, 2.0 ** 40, 2.0 ** 60])
def test_angles_of_far_positions(base, tokens):
    """The rotation of unit vectors shows the angle itself. Its fraction of a turn is known to far below 2^-32, so what is left is the
    rounding of sine and cosine (two steps at most) and of the products: 6 u."""
    rng = np.random.default_rng(tokens)
    x = np.zeros((1, 128, 1, tokens), np.float32)
    x[:, :64] = 1.0
    pos = (base * rng.uniform(0.5, 1.0, (1, 1, 1, tokens))).astype(np.float32)
    args = (x, pos, rope_frequencies(128), None, x, 1, 0, 0.0, 1.0)
    got, ref = run(rope_graph(*args))[B.NG_MODE_GRAPH_SINGLE], rope_reference(*args)
    for name in ref:
        assert np.abs(got[name] - ref[name]).max() <= 6 * U, (name, np.abs(got[name] - ref[name]).max() / U)
