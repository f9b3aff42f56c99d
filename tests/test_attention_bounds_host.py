"""The bounds of the attention tests tell apart what they are for: gradients whose operands have two fp16 parts from one."""
import numpy as np
import pytest

from attention_bounds import excess, reference_and_rss, split
from oracle import ops


def parts(t, count):
    """t in `count` fp16 parts of a common unit that takes the largest magnitude to 2^14 .. 2^15."""
    unit = 2.0 ** (14 - np.floor(np.log2(np.abs(t).max())))
    t = t * unit
    high = t.astype(np.float16).astype(np.float64)
    low = (t - high).astype(np.float16).astype(np.float64) if count == 2 else np.zeros_like(t)
    return high / unit, low / unit


def product(a, b, count):
    (ah, al), (bh, bl) = parts(a, count), parts(b, count)
    return (ah @ bh + ah @ bl + al @ bh).astype(np.float32).astype(np.float64)


def emulated(q, k, v, dy, scale, count):
    """One head: forward in fp32, every operand of a gradient's product in `count` fp16 parts."""
    p32 = ops.attention_weights(q, k, 1, 1, scale, None)[0, 0].astype(np.float32).astype(np.float64)
    Q, K, V, G = (split(t, 1)[0, 0] for t in (q, k, v, dy))
    y = (V @ p32.T).astype(np.float32).astype(np.float64)
    s = product(Q.T, K, count) * scale
    P = np.exp(s - s.max(axis=1, keepdims=True))
    P /= np.exp(scale * (Q.T @ K) - (scale * (Q.T @ K)).max(axis=1, keepdims=True)).sum(axis=1, keepdims=True)
    dS = P * (product(G.T, V, count) - (G * y).sum(axis=0)[:, None])
    return {"y": y, "dq": scale * product(K, dS.T, count), "dk": scale * product(Q, dS, count), "dv": product(G, P, count)}


@pytest.mark.parametrize("d,tq,tk", [(64, 257, 333), (96, 130, 140), (128, 300, 520), (40, 33, 31)])
def test_one_part_is_out_of_bounds_and_two_are_within(d, tq, tk):
    rng = np.random.default_rng(d)
    q, dy = (rng.standard_normal((1, d, 1, tq)).astype(np.float32) for _ in range(2))
    k, v = (rng.standard_normal((1, d, 1, tk)).astype(np.float32) for _ in range(2))
    scale = float(np.float32(d ** -0.5))
    ref, rss = reference_and_rss(q, k, v, dy, None, 1, 1, scale)
    two, one = (excess(emulated(q, k, v, dy, scale, count), ref, rss) for count in (2, 1))
    assert all(two[name] <= 1 for name in two), two
    assert all(one[name] > 2 for name in ("dq", "dk", "dv")), one
