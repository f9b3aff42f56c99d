"""Graphs of attention operators for the tests: one operator with its gradients, every tensor an output."""
import numpy as np

import workloads
from oracle import ops
from oracle.backward import attention_vjp, head_rope_vjp


class Graph:
    """Nodes of a workload by name."""

    def __init__(self):
        self.nodes, self.inputs, self.names = [], {}, {}

    def given(self, name, value):
        value = np.ascontiguousarray(value, dtype=np.float32)
        self.inputs[len(self.nodes)] = value
        return self._add(name, workloads.Node("input", [], dict(zip("nchw", value.shape)), [], value.shape))

    def node(self, name, op, preds, shape=(0, 0, 0, 0), weights=(), shared=(), **params):
        preds = [self.names[p] if isinstance(p, str) else p for p in preds]
        return self._add(name, workloads.Node(op, preds, params, list(weights), tuple(shape), 1.0, list(shared)))

    def _add(self, name, nd):
        self.nodes.append(nd)
        self.names[name] = len(self.nodes) - 1
        return len(self.nodes) - 1

    def workload(self):
        outputs = [v for v, nd in enumerate(self.nodes) if nd.op != "input"]
        return workloads.Workload("attention", self.nodes, self.inputs[0], outputs, inputs=self.inputs)


def attention_graph(q, k, v, dy, lengths, heads, kv_heads, scale):
    g = Graph()
    for name, t in (("q", q), ("k", k), ("v", v), ("dy", dy)):
        g.given(name, t)
    last = []
    if lengths is not None:
        g.given("lengths", lengths)
        last = ["lengths"]
    how = dict(heads=heads, kv_heads=kv_heads, scale=scale)
    g.node("y", "attention", ["q", "k", "v"] + last, np.shape(q), **how)
    if dy is not None:
        g.node("rows", "attention_rows", ["dy", "y"], heads=heads)
        for name in ("dq", "dk", "dv"):
            g.node(name, "attention_" + name, ["dy", "rows", "q", "k", "v"] + last, **how)
    return g


def attention_reference(q, k, v, dy, lengths, heads, kv_heads, scale):
    """In 64 bits: y, dq, dk, dv."""
    scale = float(np.float32(scale))
    p = ops.attention_weights(q, k, heads, kv_heads, scale, lengths)
    vh = ops.counted_values(v, kv_heads, lengths)
    y = np.stack([np.stack([vh[b, h // (heads // kv_heads)] @ p[b, h].T for h in range(heads)]) for b in range(p.shape[0])]).reshape(np.shape(q))
    return dict(zip(("y", "dq", "dk", "dv"), (y,) + attention_vjp(q, k, v, lengths, heads, kv_heads, scale, dy)))


def rope_graph(x, pos, freq, gamma, dy, heads, interleaved, eps, factor):
    g = Graph()
    for name, t in (("x", x), ("pos", pos), ("dy", dy)):
        g.given(name, t)
    weights = [freq] + ([gamma] if gamma is not None else [])
    how = dict(heads=heads, rot=2 * len(freq), interleaved=interleaved, eps=eps, factor=factor)
    y = g.node("y", "head_rope", ["x", "pos"], np.shape(x), weights, **how)
    shared = [(y, j) for j in range(len(weights))]
    g.node("dx", "head_rope_dgrad", ["dy", "x", "pos"], shared=shared, **how)
    if gamma is not None:
        g.node("dgamma", "head_rope_wgrad", ["dy", "x", "pos"], shared=shared, **how)
    return g


def rope_reference(x, pos, freq, gamma, dy, heads, interleaved, eps, factor):
    f64 = lambda t: None if t is None else np.asarray(t, dtype=np.float64)  # noqa: E731
    keep, ops._out = ops._out, f64
    try:
        y = ops.head_rope(x, pos, freq, gamma, heads, bool(interleaved), float(np.float32(eps)), float(np.float32(factor)))
    finally:
        ops._out = keep
    dx, dg = head_rope_vjp(x, pos, freq, gamma, heads, bool(interleaved), float(np.float32(eps)), float(np.float32(factor)), dy)
    out = {"y": y, "dx": dx}
    if gamma is not None:
        out["dgamma"] = dg.reshape(1, -1, 1, 1)
    return out
