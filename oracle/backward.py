"""Gradients of a DAG for the oracle (test infrastructure, see package doc).

Section 5 of the paper ("Training", the batch-32 training throughput figure)
replays a whole training iteration - forward pass, backward pass and weight
update - as one recorded schedule; what is computed is the framework's ordinary
backward pass. This module states that computation once, plainly: for the scalar

    L = sum over output nodes o of  <value[o], seed[o]>

it returns dL/d(value[v]) for every node and dL/d(weight) for every weight
tensor, each operator by the textbook vector-Jacobian product of the formula
in module ``ops``, nodes visited in descending id, fp64 arithmetic throughout.

Readings (the paper does not go below "the framework's backward pass"):
* batch norm keeps its statistics fixed (the inference-form affine map of
  ``ops.bn_act``), so gamma and beta get gradients, mean and var do not;
* a max pool sends the gradient to the first tap, in row-major window order,
  that attains the maximum; an average pool divides by the number of in-bounds
  taps, as the forward pass does;
* activations that the backward pass reads are the forward pass's stored values.

Parity status: pinned against central finite differences of an fp64 forward
pass on tiny DAGs and against torch.autograd (CPU, fp64) operator by operator.
No HIP counterpart exists yet: nothing on the GPU is compared with this module.
"""
from __future__ import annotations

from typing import Dict, List, Optional, Tuple

import numpy as np

from . import ops
from .forward import eval_node, input_value


def _f64(x):
    return np.asarray(x, dtype=np.float64)


def _taps(k, stride, ho, wo):
    for a in range(k):
        for b in range(k):
            yield a, b, (slice(None), slice(None),
                         slice(a, a + stride * (ho - 1) + 1, stride), slice(b, b + stride * (wo - 1) + 1, stride))


def _unpad(xp, pad):
    return xp[:, :, pad:xp.shape[2] - pad, pad:xp.shape[3] - pad] if pad else xp


def conv2d_vjp(x, w, stride, pad, dy):
    """y[n,o,i,j] = sum w[o,c,a,b] xp[n,c,i s+a,j s+b]  =>
    dxp[n,c,i s+a,j s+b] += sum_o w[o,c,a,b] dy[n,o,i,j];  dw[o,c,a,b] = sum_{n,i,j} dy[n,o,i,j] xp[n,c,i s+a,j s+b]."""
    x, w, dy = _f64(x), _f64(w), _f64(dy)
    n, c, h, wd = x.shape
    o, _, k, _ = w.shape
    ho, wo = dy.shape[2], dy.shape[3]
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)))
    dxp = np.zeros_like(xp)
    dw = np.zeros_like(w)
    dyf = dy.reshape(n, o, ho * wo)
    for a, b, sl in _taps(k, stride, ho, wo):
        dxp[sl] += np.matmul(w[:, :, a, b].T[None], dyf).reshape(n, c, ho, wo)
        dw[:, :, a, b] = np.einsum("nop,ncp->oc", dyf, xp[sl].reshape(n, c, ho * wo))
    return _unpad(dxp, pad), dw


def dwconv_vjp(x, w, stride, dy):
    x, w, dy = _f64(x), _f64(w), _f64(dy)
    k = w.shape[1]
    pad = k // 2
    ho, wo = dy.shape[2], dy.shape[3]
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)))
    dxp = np.zeros_like(xp)
    dw = np.zeros_like(w)
    for a, b, sl in _taps(k, stride, ho, wo):
        dxp[sl] += w[None, :, a, b, None, None] * dy
        dw[:, a, b] = (dy * xp[sl]).sum(axis=(0, 2, 3))
    return _unpad(dxp, pad), dw


def bn_act_vjp(x, gamma, beta, mean, var, eps, relu, dy):
    x, dy = _f64(x), _f64(dy)
    g, b, m, v = (_f64(t)[None, :, None, None] for t in (gamma, beta, mean, var))
    xhat = (x - m) / np.sqrt(v + eps)
    if relu:
        dy = dy * (g * xhat + b > 0.0)
    return dy * g / np.sqrt(v + eps), (dy * xhat).sum(axis=(0, 2, 3)), dy.sum(axis=(0, 2, 3))


def pool3x3_vjp(x, mode, stride, pad, dy):
    x, dy = _f64(x), _f64(dy)
    n, c, h, w = x.shape
    ho, wo = dy.shape[2], dy.shape[3]
    fill = -np.inf if mode == "max" else 0.0
    xp = np.pad(x, ((0, 0), (0, 0), (pad, pad), (pad, pad)), constant_values=fill)
    dxp = np.zeros_like(xp)
    if mode == "max":
        best = np.full((n, c, ho, wo), -np.inf)
        for a, b, sl in _taps(3, stride, ho, wo):
            best = np.maximum(best, xp[sl])
        taken = np.zeros((n, c, ho, wo), dtype=bool)
        for a, b, sl in _taps(3, stride, ho, wo):
            hit = (xp[sl] == best) & ~taken
            dxp[sl] += dy * hit
            taken |= hit
    else:
        ones = np.pad(np.ones((1, 1, h, w)), ((0, 0), (0, 0), (pad, pad), (pad, pad)))
        cnt = np.zeros((1, 1, ho, wo))
        for a, b, sl in _taps(3, stride, ho, wo):
            cnt = cnt + ones[sl]
        for a, b, sl in _taps(3, stride, ho, wo):
            dxp[sl] += dy / cnt * ones[sl]
    return _unpad(dxp, pad)


def head_rope_vjp(x, positions, freq, gamma, heads, interleaved, eps, factor, dy):
    """The rotation's transpose takes dy back to du; through u = gamma x / rms: dx = (gamma du - xh mean(gamma du xh)) / rms with
    xh = x / rms, dgamma = sum du xh. (dx, dgamma or None); no gradient goes to the positions."""
    x, dy = _f64(x), _f64(dy)
    n, c, h, w = x.shape
    shape = (n, heads, c // heads, h * w)
    x, g = x.reshape(shape), dy.reshape(shape)
    t = ops.rope_angles(positions, freq, n)[:, None]
    ia, ib = ops.rope_pair_channels(2 * len(freq), interleaved)
    du = g.copy()
    du[:, :, ia] = factor * (g[:, :, ia] * np.cos(t) + g[:, :, ib] * np.sin(t))
    du[:, :, ib] = factor * (g[:, :, ib] * np.cos(t) - g[:, :, ia] * np.sin(t))
    if gamma is None:
        return du.reshape(n, c, h, w), None
    rms = np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    xh = x / rms
    gu = du * _f64(gamma)[None, None, :, None]
    dx = (gu - xh * (gu * xh).mean(axis=2, keepdims=True)) / rms
    return dx.reshape(n, c, h, w), (du * xh).sum(axis=(0, 1, 3))


def attention_vjp(q, k, v, lengths, heads, kv_heads, scale, dy):
    """dv = p^T dy; ds = p (dp - <p, dp>) with dp = <dy, v>; dq = scale ds k, dk = scale ds^T q; heads that share a key head add up."""
    p = ops.attention_weights(q, k, heads, kv_heads, scale, lengths)
    n, group = p.shape[0], heads // kv_heads
    qh, gh = (_f64(t).reshape(n, heads, -1, p.shape[2]) for t in (q, dy))
    kh, vh = (ops.counted_values(t, kv_heads, lengths) for t in (k, v))
    dq, dk, dv = np.zeros_like(qh), np.zeros_like(kh), np.zeros_like(vh)
    for b in range(n):
        for h in range(heads):
            j = h // group
            dv[b, j] += gh[b, h] @ p[b, h]
            dp = gh[b, h].T @ vh[b, j]
            ds = p[b, h] * (dp - (p[b, h] * dp).sum(axis=1, keepdims=True))
            dq[b, h] = scale * (kh[b, j] @ ds.T)
            dk[b, j] += scale * (qh[b, h] @ ds)
    return dq.reshape(np.shape(q)), dk.reshape(np.shape(k)), dv.reshape(np.shape(v))


def node_vjp(nd, ins, dy) -> Tuple[List[np.ndarray], List[np.ndarray]]:
    """(gradients w.r.t. the node's inputs, gradients w.r.t. its weight tensors)."""
    p, w = nd.params, nd.weights
    if nd.op == "conv1x1":
        dx, dw = conv2d_vjp(ins[0], _f64(w[0])[:, :, None, None], 1, 0, dy)
        return [dx], [dw[:, :, 0, 0]]
    if nd.op == "conv3x3":
        dx, dw = conv2d_vjp(ins[0], w[0], p["stride"], p["pad"], dy)
        return [dx], [dw]
    if nd.op == "dwconv":
        dx, dw = dwconv_vjp(ins[0], w[0], p["stride"], dy)
        return [dx], [dw]
    if nd.op == "bn_act":
        dx, dg, db = bn_act_vjp(ins[0], w[0], w[1], w[2], w[3], p["eps"], bool(p["relu"]), dy)
        return [dx], [dg, db, np.zeros_like(dg), np.zeros_like(dg)]
    if nd.op == "relu":
        return [_f64(dy) * (_f64(ins[0]) > 0.0)], []
    if nd.op == "add_n":
        return [_f64(dy).copy() for _ in ins], []
    if nd.op == "concat":
        out, first = [], 0
        for t, lo, hi in zip(ins, p["lo"], p["hi"]):
            d = np.zeros(t.shape)
            d[:, lo:hi] = _f64(dy)[:, first:first + hi - lo]
            first += hi - lo
            out.append(d)
        return out, []
    if nd.op == "pool":
        return [pool3x3_vjp(ins[0], p["mode"], p["stride"], p["pad"], dy)], []
    if nd.op == "global_avgpool":
        h, wd = ins[0].shape[2], ins[0].shape[3]
        return [np.broadcast_to(_f64(dy) / (h * wd), ins[0].shape).copy()], []
    if nd.op == "fc":
        x, dyf = _f64(ins[0]).reshape(ins[0].shape[0], -1), _f64(dy).reshape(dy.shape[0], -1)
        return [(dyf @ _f64(w[0])).reshape(ins[0].shape)], [dyf.T @ x, dyf.sum(axis=0)]
    if nd.op == "head_rope":
        dx, dg = head_rope_vjp(ins[0], ins[1], w[0], w[1] if len(w) > 1 else None, p["heads"], bool(p["interleaved"]), p["eps"], p["factor"], dy)
        return [dx, np.zeros(ins[1].shape)], [np.zeros(len(w[0]))] + ([dg] if dg is not None else [])
    if nd.op == "attention":
        lengths = ins[3] if len(ins) > 3 else None
        grads = attention_vjp(ins[0], ins[1], ins[2], lengths, p["heads"], p["kv_heads"], p["scale"], dy)
        return list(grads) + ([np.zeros(lengths.shape)] if lengths is not None else []), []
    raise ValueError(f"unknown op {nd.op!r}")


def backward(workload, seed: Dict[int, np.ndarray], x: Optional[np.ndarray] = None):
    """Returns (d_value, d_weight): d_value[v] = dL/d(value of node v) for every node,
    d_weight[v] = list of dL/d(weight j of node v), for L = sum_o <value[o], seed[o]>."""
    nodes = workload.nodes
    x = workload.input if x is None else x
    val: Dict[int, np.ndarray] = {}
    for v, nd in enumerate(nodes):
        val[v] = np.asarray(input_value(workload, v, x)) if nd.op == "input" else eval_node(nd, [val[u] for u in nd.preds])
    d_value = {v: np.zeros(val[v].shape) for v in range(len(nodes))}
    d_weight: Dict[int, List[np.ndarray]] = {}
    for o, s in seed.items():
        d_value[o] = d_value[o] + _f64(s)
    for v in range(len(nodes) - 1, -1, -1):
        nd = nodes[v]
        if nd.op == "input":
            continue
        dins, dws = node_vjp(nd, [val[u] for u in nd.preds], d_value[v])
        for u, d in zip(nd.preds, dins):          # a tensor read twice by one node gets both contributions
            d_value[u] = d_value[u] + d
        d_weight[v] = dws
    return d_value, d_weight


def sgd_step(weights: List[np.ndarray], grads: List[np.ndarray], lr: float) -> List[np.ndarray]:
    """Plain stochastic gradient descent: w <- w - lr * dL/dw, in fp64, stored as fp32."""
    return [np.ascontiguousarray(_f64(w) - lr * _f64(g), dtype=np.float32) for w, g in zip(weights, grads)]
