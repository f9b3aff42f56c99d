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


def distances(tq: int, tk: int, reach: int, offset: int):
    """[query][key]: place of the distance j - (i + offset) in a bias of the distances -reach .. reach; farther ones are taken as these."""
    d = np.arange(tk)[None, :] - (np.arange(tq)[:, None] + offset)
    return np.clip(d, -reach, reach) + reach


def attention_weights(q, k, heads: int, kv_heads: int, scale: float, lengths, bias=None, at: str = "first"):
    """p[n][head][query][key]: softmax over the keys that count (and, with a bias, are seen: not -infinity), 0 for the others (and everywhere
    for a query without any). ``at``: the bias counts distances from the first key ("first") or so that the last query is at the last
    key that counts ("last")."""
    q, k = _f64(q), _f64(k)
    n, c = q.shape[:2]
    q, k = q.reshape(n, heads, c // heads, -1), k.reshape(n, kv_heads, c // heads, -1)
    tq, tk = q.shape[3], k.shape[3]
    p = np.zeros((n, heads, tq, tk))
    for b in range(n):
        m = tk if lengths is None else key_count(float(np.ravel(lengths)[b]), tk)
        for h in range(heads if m else 0):
            s = scale * (q[b, h].T @ k[b, h // (heads // kv_heads)][:, :m])
            if bias is not None:
                row = _f64(bias).reshape(heads, -1)[h]
                s = s + row[distances(tq, m, len(row) // 2, m - tq if at == "last" else 0)]
            top = s.max(axis=1, keepdims=True)
            e = np.exp(s - np.where(np.isneginf(top), 0.0, top))
            total = e.sum(axis=1, keepdims=True)
            p[b, h, :, :m] = e / np.where(total == 0.0, 1.0, total)
    return p


def counted_values(v, kv_heads: int, lengths):
    """v by heads, zeros in the place of what does not count."""
    v = _f64(v)
    v = v.reshape(v.shape[0], kv_heads, v.shape[1] // kv_heads, -1).copy()
    for b in range(v.shape[0] if lengths is not None else 0):
        v[b, :, :, key_count(float(np.ravel(lengths)[b]), v.shape[3]):] = 0.0
    return v


def attention(q, k, v, lengths, heads: int, kv_heads: int, scale: float, bias=None, at: str = "first"):
    """y[query] = sum over keys p[query][key] v[key]."""
    p = attention_weights(q, k, heads, kv_heads, scale, lengths, bias, at)
    vh = counted_values(v, kv_heads, lengths)
    y = np.stack([np.stack([vh[b, h // (heads // kv_heads)] @ p[b, h].T for h in range(heads)]) for b in range(p.shape[0])])
    return _out(y.reshape(q.shape))


def layer_norm(x, gamma, beta, eps: float):
    """gamma (x - mean) / sqrt(variance + eps) + beta over the channels of each pixel."""
    x = _f64(x)
    centred = x - x.mean(axis=1, keepdims=True)
    xh = centred / np.sqrt((centred * centred).mean(axis=1, keepdims=True) + eps)
    return _out(xh * _f64(gamma)[None, :, None, None] + _f64(beta)[None, :, None, None])


def philox4x32(counter, key):
    """Ten rounds of Philox4x32 (Salmon et al., SC 2011) on counters [m][4] with a key of two words: [m][4] words."""
    c = [counter[:, j].astype(np.uint64) for j in range(4)]
    k = [int(key[0]), int(key[1])]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).astype(np.uint32)


def dropout_scale(shape, seed, rate: float, site: int):
    """What each element is multiplied by: 1 / (1 - rate) where it is kept, 0 where it is dropped (rate rounded to 2^-32)."""
    total = int(np.prod(shape))
    e = np.arange((total + 3) // 4, dtype=np.uint64)
    counter = np.stack([e & np.uint64(0xFFFFFFFF), e >> np.uint64(32), np.full_like(e, site), np.zeros_like(e)], 1)
    words = philox4x32(counter, np.ascontiguousarray(seed, dtype=np.float32).reshape(2).view(np.uint32)).ravel()[:total]
    limit = int(np.rint(float(np.float32(rate)) * 2.0 ** 32))
    return np.where(words.astype(np.int64) >= limit, 2.0 ** 32 / (2.0 ** 32 - limit), 0.0).reshape(shape)


def dropout(x, seed, residual, rate: float, site: int):
    m = dropout_scale(np.shape(x), seed, rate, site)
    y = np.where(m > 0, _f64(x) * m, 0.0) if m.size else m
    return _out(y if residual is None else _f64(residual) + y)


def position_bucket(distance: int, buckets: int, max_distance: int, both: bool):
    """Bucket of a distance (key less query), None for keys behind the query where they are not seen. In whole numbers: step j of the
    logarithmic buckets is reached where (|d| / exact)^steps >= (max_distance / exact)^j."""
    b = buckets // 2 if both else buckets
    exact, far = b // 2, abs(distance)
    if distance > 0 and not both:
        return None
    if far >= exact:
        steps = b - exact
        j = 0
        while j < steps and far ** steps * exact ** (j + 1) >= max_distance ** (j + 1) * exact ** steps:
            j += 1
        far = min(exact + j, b - 1)
    return far + (b if distance > 0 else 0)


def position_bias(table, heads: int, buckets: int, max_distance: int, both: bool):
    table = _f64(table).reshape(buckets, heads)
    of = [position_bucket(d, buckets, max_distance, both) for d in range(-max_distance, max_distance + 1)]
    return _out(np.stack([np.full(heads, -np.inf) if b is None else table[b] for b in of], 1).reshape(1, heads, 1, -1))
