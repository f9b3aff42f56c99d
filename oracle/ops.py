"""Operator definitions for the oracle (test infrastructure, see package doc).

The paper runs unchanged framework operators (Section 5, "Experimental
Setup"): what a task computes is the standard inference-time definition of
each layer. Every function takes/returns fp32 NCHW arrays and does its
arithmetic in fp64. No blocking, no fusion: one formula per function.
"""
from __future__ import annotations

import numpy as np


def _f64(x):
    return np.asarray(x, dtype=np.float64)


def _out(x):
    return np.ascontiguousarray(x, dtype=np.float32)


def out_size(size: int, k: int, stride: int, pad: int) -> int:
    """Number of window positions along one axis."""
    return (size + 2 * pad - k) // stride + 1


def conv2d(x, w, stride: int, pad: int):
    """Dense cross-correlation: y[n,o,i,j] = sum_{c,a,b} w[o,c,a,b] * xp[n,c,i*s+a,j*s+b],
    xp = x zero-padded by ``pad`` on each spatial side."""
    x, w = _f64(x), _f64(w)
    n, c, h, wd = x.shape
    o, c2, k, k2 = w.shape
    assert c == c2 and k == k2
    ho, wo = out_size(h, k, stride, pad), out_size(wd, k, stride, pad)
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)))
    y = np.zeros((n, o, ho, wo))
    for a in range(k):
        for b in range(k):
            tap = xp[:, :, a:a + stride * (ho - 1) + 1:stride, b:b + stride * (wo - 1) + 1:stride]
            # contraction over input channels for this tap (a matmul per image)
            y += np.matmul(w[:, :, a, b][None], tap.reshape(n, c, ho * wo)).reshape(n, o, ho, wo)
    return _out(y)


def conv1x1(x, w):
    """Pointwise convolution: y[n,o,i,j] = sum_c w[o,c] * x[n,c,i,j]."""
    w = _f64(w)
    return conv2d(x, w[:, :, None, None], 1, 0)


def conv3x3(x, w, stride: int, pad: int):
    return conv2d(x, w, stride, pad)


def dwconv(x, w, stride: int):
    """Depthwise k x k, pad k//2: y[n,c,i,j] = sum_{a,b} w[c,a,b] * xp[n,c,i*s+a,j*s+b]."""
    x, w = _f64(x), _f64(w)
    n, c, h, wd = x.shape
    c2, k, k2 = w.shape
    assert c == c2 and k == k2
    pad = k // 2
    ho, wo = out_size(h, k, stride, pad), out_size(wd, k, stride, pad)
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)))
    y = np.zeros((n, c, ho, wo))
    for a in range(k):
        for b in range(k):
            tap = xp[:, :, a:a + stride * (ho - 1) + 1:stride, b:b + stride * (wo - 1) + 1:stride]
            y += w[None, :, a, b, None, None] * tap
    return _out(y)


def bn_act(x, gamma, beta, mean, var, eps: float, relu: bool):
    """Inference batch norm: y = gamma * (x - mean) / sqrt(var + eps) + beta, then optional max(.,0)."""
    x = _f64(x)
    g, b, m, v = (_f64(t)[None, :, None, None] for t in (gamma, beta, mean, var))
    y = g * (x - m) / np.sqrt(v + eps) + b
    if relu:
        y = np.maximum(y, 0.0)
    return _out(y)


def relu(x):
    return _out(np.maximum(_f64(x), 0.0))


def add_n(xs):
    """Elementwise sum, accumulated left to right."""
    y = _f64(xs[0]).copy()
    for t in xs[1:]:
        assert t.shape == xs[0].shape
        y += _f64(t)
    return _out(y)


def concat(xs, lo, hi):
    """Stack channel slices xs[j][:, lo[j]:hi[j]] along C, in order."""
    return _out(np.concatenate([_f64(t)[:, l:h] for t, l, h in zip(xs, lo, hi)], axis=1))


def pool3x3(x, mode: str, stride: int, pad: int):
    """3x3 window. 'max': maximum over in-bounds taps. 'avg': sum of in-bounds taps
    divided by their count (padding is excluded from the divisor)."""
    x = _f64(x)
    n, c, h, w = x.shape
    ho, wo = out_size(h, 3, stride, pad), out_size(w, 3, stride, pad)
    fill = -np.inf if mode == "max" else 0.0
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)), constant_values=fill)
    ones = np.pad(np.ones((1, 1, h, w)), ((0, 0), (0, 0), (pad, pad), (pad, pad)))
    acc = np.full((n, c, ho, wo), fill)
    cnt = np.zeros((1, 1, ho, wo))
    for a in range(3):
        for b in range(3):
            sl = (slice(None), slice(None),
                  slice(a, a + stride * (ho - 1) + 1, stride), slice(b, b + stride * (wo - 1) + 1, stride))
            if mode == "max":
                acc = np.maximum(acc, xp[sl])
            else:
                acc = acc + xp[sl]
                cnt = cnt + ones[sl]
    return _out(acc if mode == "max" else acc / cnt)


def global_avgpool(x):
    return _out(_f64(x).mean(axis=(2, 3), keepdims=True))


def fc(x, w, b):
    """y[n,o] = sum_c w[o,c] * x[n,c] + b[o], on [n,c,1,1] tensors."""
    x, w, b = _f64(x), _f64(w), _f64(b)
    n, c, h, wd = x.shape
    assert h == 1 and wd == 1
    return _out((x.reshape(n, c) @ w.T + b[None]).reshape(n, -1, 1, 1))


def rope_angles(positions, freq, n):
    """[n, rot / 2, tokens]: angle of every pair at every token."""
    pos = _f64(positions).reshape(np.shape(positions)[0], 1, -1)
    return np.broadcast_to(pos * _f64(freq)[None, :, None], (n, len(freq), pos.shape[2]))


def rope_pair_channels(rot: int, interleaved: bool):
    """First and second channels of the rotated pairs of a head."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def head_rope(x, positions, freq, gamma, heads: int, interleaved: bool, eps: float, factor: float):
    """Each head (a run of channels): x gamma / sqrt(mean x^2 + eps) (gamma None: x), then its first 2 len(freq) channels rotated in
    pairs by position * freq and multiplied by factor."""
    x = _f64(x)
    n, c, h, w = x.shape
    u = x.reshape(n, heads, c // heads, h * w)
    if gamma is not None:
        u = u / np.sqrt((u * u).mean(axis=2, keepdims=True) + eps) * _f64(gamma)[None, None, :, None]
    y = u.copy()
    t = rope_angles(positions, freq, n)[:, None]
    ia, ib = rope_pair_channels(2 * len(freq), interleaved)
    y[:, :, ia] = factor * (u[:, :, ia] * np.cos(t) - u[:, :, ib] * np.sin(t))
    y[:, :, ib] = factor * (u[:, :, ia] * np.sin(t) + u[:, :, ib] * np.cos(t))
    return _out(y.reshape(n, c, h, w))


def key_count(length, tk: int) -> int:
    """Keys j < length; none if it is not a number."""
    return sum(1 for j in range(tk) if j < length)


def attention_weights(q, k, heads: int, kv_heads: int, scale: float, lengths):
    """p[n][head][query][key]: softmax over the keys that count, 0 for the others (and everywhere for an image without any)."""
    q, k = _f64(q), _f64(k)
    n, c = q.shape[:2]
    q, k = q.reshape(n, heads, c // heads, -1), k.reshape(n, kv_heads, c // heads, -1)
    p = np.zeros((n, heads, q.shape[3], k.shape[3]))
    for b in range(n):
        m = k.shape[3] if lengths is None else key_count(float(np.ravel(lengths)[b]), k.shape[3])
        for h in range(heads if m else 0):
            s = scale * (q[b, h].T @ k[b, h // (heads // kv_heads)][:, :m])
            e = np.exp(s - s.max(axis=1, keepdims=True))
            p[b, h, :, :m] = e / e.sum(axis=1, keepdims=True)
    return p


def counted_values(v, kv_heads: int, lengths):
    """v by heads, zeros in the place of what does not count."""
    v = _f64(v)
    v = v.reshape(v.shape[0], kv_heads, v.shape[1] // kv_heads, -1).copy()
    for b in range(v.shape[0] if lengths is not None else 0):
        v[b, :, :, key_count(float(np.ravel(lengths)[b]), v.shape[3]):] = 0.0
    return v


def attention(q, k, v, lengths, heads: int, kv_heads: int, scale: float):
    """y[query] = sum over keys p[query][key] v[key]."""
    p = attention_weights(q, k, heads, kv_heads, scale, lengths)
    vh = counted_values(v, kv_heads, lengths)
    y = np.stack([np.stack([vh[b, h // (heads // kv_heads)] @ p[b, h].T for h in range(heads)]) for b in range(p.shape[0])])
    return _out(y.reshape(q.shape))
