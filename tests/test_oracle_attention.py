"""Pins of the oracle's attention operators: torch in 64 bits for the values and the gradients, central differences for the
gradients, and the rules for keys that do not count."""
import numpy as np
import pytest
import torch

from oracle import ops
from oracle.backward import attention_vjp, head_rope_vjp
from workloads import rope_frequencies


@pytest.fixture(autouse=True)
def fp64_storage(monkeypatch):
    monkeypatch.setattr(ops, "_out", lambda x: np.ascontiguousarray(x, dtype=np.float64))


def _torch_rope(x, pos, freq, gamma, heads, interleaved, eps, factor):
    n, c, h, w = x.shape
    u = x.reshape(n, heads, c // heads, h * w)
    if gamma is not None:
        u = u / (u.pow(2).mean(2, keepdim=True) + eps).sqrt() * gamma[None, None, :, None]
    rot = 2 * len(freq)
    t = (pos.reshape(-1, 1, h * w) * freq[None, :, None])[:, None]
    head = u[:, :, :rot]
    a, b = (head[:, :, 0::2], head[:, :, 1::2]) if interleaved else head.chunk(2, 2)
    z = torch.complex(a, b) * torch.polar(torch.full_like(t, factor), t)
    turned = torch.stack([z.real, z.imag], 3).flatten(2, 3) if interleaved else torch.cat([z.real, z.imag], 2)
    return torch.cat([turned, u[:, :, rot:]], 2).reshape(n, c, h, w)


def _torch_attention(q, k, v, lengths, heads, kv_heads, scale):
    n, c = q.shape[:2]
    d = c // heads
    out = []
    for b in range(n):
        m = k[b].reshape(kv_heads * d, -1).shape[1] if lengths is None else lengths[b]
        qb = q[b].reshape(heads, d, -1)
        kb, vb = (t[b].reshape(kv_heads, d, -1)[:, :, :m].repeat_interleave(heads // kv_heads, 0) for t in (k, v))
        if m == 0:
            out.append(torch.zeros_like(qb))
        else:
            out.append((torch.softmax(scale * qb.transpose(1, 2) @ kb, 2) @ vb.transpose(1, 2)).transpose(1, 2))
    return torch.stack(out).reshape(q.shape)


@pytest.mark.parametrize("interleaved", [0, 1])
@pytest.mark.parametrize("norm,rot,d", [(1, 8, 8), (1, 4, 7), (0, 6, 9), (0, 2, 2)])
def test_head_rope_and_its_gradients(interleaved, norm, rot, d):
    rng = np.random.default_rng(1)
    n, heads, h, w = 2, 3, 2, 5
    x, dy = rng.standard_normal((2, n, heads * d, h, w))
    pos = rng.integers(0, 5000, (n, 1, h, w)).astype(np.float64)
    freq = rope_frequencies(rot).astype(np.float64)
    gamma = rng.uniform(0.5, 1.5, d) if norm else None
    got = ops.head_rope(x, pos, freq, gamma, heads, bool(interleaved), 1e-5, 1.25)
    xt = torch.tensor(x, requires_grad=True)
    gt = torch.tensor(gamma, requires_grad=True) if norm else None
    ref = _torch_rope(xt, torch.tensor(pos), torch.tensor(freq), gt, heads, bool(interleaved), 1e-5, 1.25)
    np.testing.assert_allclose(got, ref.detach().numpy(), rtol=0, atol=1e-11)
    ref.backward(torch.tensor(dy))
    dx, dg = head_rope_vjp(x, pos, freq, gamma, heads, bool(interleaved), 1e-5, 1.25, dy)
    np.testing.assert_allclose(dx, xt.grad.numpy(), rtol=0, atol=1e-10)
    if norm:
        np.testing.assert_allclose(dg, gt.grad.numpy(), rtol=0, atol=1e-9)
    else:
        assert dg is None


@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (4, 2), (3, 1)])
@pytest.mark.parametrize("lengths", [None, (7, 0, 3)])
def test_attention_and_its_gradients(heads, kv_heads, lengths):
    rng = np.random.default_rng(2)
    n, d, tq, tk, scale = 3, 5, 4, 7, 0.6
    q, dy = rng.standard_normal((2, n, heads * d, 1, tq))
    k, v = rng.standard_normal((2, n, kv_heads * d, 1, tk))
    ln = None if lengths is None else np.array(lengths, np.float64).reshape(n, 1, 1, 1)
    t = [torch.tensor(a, requires_grad=True) for a in (q, k, v)]
    ref = _torch_attention(*t, lengths, heads, kv_heads, scale)
    np.testing.assert_allclose(ops.attention(q, k, v, ln, heads, kv_heads, scale), ref.detach().numpy(), rtol=0, atol=1e-13)
    ref.backward(torch.tensor(dy))
    for got, a in zip(attention_vjp(q, k, v, ln, heads, kv_heads, scale, dy), t):
        np.testing.assert_allclose(got, a.grad.numpy(), rtol=0, atol=1e-12)
    # central differences of <y, dy>
    grads = attention_vjp(q, k, v, ln, heads, kv_heads, scale, dy)
    for j, a in enumerate((q, k, v)):
        for at in [tuple(rng.integers(0, s) for s in a.shape) for _ in range(4)]:
            keep, step, side = a[at], 1e-6, []
            for sgn in (1, -1):
                a[at] = keep + sgn * step
                side.append((ops.attention(q, k, v, ln, heads, kv_heads, scale) * dy).sum())
            a[at] = keep
            assert abs((side[0] - side[1]) / (2 * step) - grads[j][at]) < 1e-7


def test_what_does_not_count_is_not_looked_at():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((3, 2, 6, 1, 5))
    ln = np.array([2.0, np.nan]).reshape(2, 1, 1, 1)
    ref = ops.attention(q, k, v, ln, 2, 2, 0.5)
    k[0, :, :, 2:], v[0, :, :, 2:], k[1], v[1] = np.nan, np.inf, np.nan, np.nan
    got = ops.attention(q, k, v, ln, 2, 2, 0.5)
    assert np.array_equal(got, ref) and not got[1].any() and np.isfinite(got).all()
    assert [ops.key_count(x, 5) for x in (-1.0, 0.0, 0.5, 3.0, 5.0, 1e9, float("nan"))] == [0, 0, 1, 3, 5, 5, 0]


def test_scaled_frequencies():
    plain = rope_frequencies(64)
    assert plain[0] == 1 and plain.shape == (32,)
    np.testing.assert_allclose(rope_frequencies(64, scaling="linear", factor=4.0), plain / 4, rtol=1e-6)
    ntk = rope_frequencies(64, scaling="ntk", factor=4.0)
    assert ntk[0] == 1 and abs(ntk[-1] / plain[-1] - 0.25) < 1e-5
    with pytest.raises(ValueError):
        rope_frequencies(8, scaling="other")
