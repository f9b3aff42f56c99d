"""Graphs of the operators around the attention of a transformer block, run in the replay modes, and bounds of their errors."""
import numpy as np

from attention_util import Graph
from oracle import ops
from oracle.backward import layer_norm_vjp
from paper_2012_02732_amd import GraphRunner, binding as B

U = 2.0 ** -24                                                   # half a step of fp32
MODES = (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_SINGLE, B.NG_MODE_EAGER_MULTI, B.NG_MODE_DEVICE_RESIDENT)


def run(g, modes=(B.NG_MODE_GRAPH_SINGLE,), replays=1, device="cuda:0", **prepare):
    """{mode: {name: tensor}}; a mode without a plan is left out. Every replay starts from an arena that holds NaN."""
    r = GraphRunner(g.workload(), device)
    try:
        r.prepare(plan_trials=1, **prepare)
        got = {}
        for mode in modes:
            for turn in range(replays):
                r.arena.fill_(0xFF)
                for v, t in g.inputs.items():
                    r.set_input(t, v)
                try:
                    r.replay(mode)
                except B.NgError as e:
                    assert mode in (B.NG_MODE_DEVICE_RESIDENT, B.NG_MODE_GRAPH_MULTI) and e.code == B.NG_ESTATE, (mode, e)
                    break
                r.sync()
                now = {name: r.output(v) for name, v in g.names.items() if v not in g.inputs}
                if turn:
                    assert all(np.array_equal(got[mode][name], t, equal_nan=True) for name, t in now.items()), (mode, turn)
                got[mode] = now
        return got
    finally:
        r.close()


def kernels(g):
    """Name of the kernel of each node."""
    r = GraphRunner(g.workload())
    try:
        r.schedule(), r.plan()
        return {name: B.ng_planned_task_kernel(r.g, v) for name, v in g.names.items() if v not in g.inputs}
    finally:
        r.close()


def norm_graph(x, gamma, beta, dy, eps, both=True):
    g = Graph()
    g.given("x", x)
    y = g.node("y", "layer_norm", ["x"], np.shape(x), [gamma, beta], eps=eps)
    if dy is not None:
        g.given("dy", dy)
        g.node("dx", "layer_norm_dgrad", ["dy", "x"], shared=[(y, 0), (y, 1)], eps=eps)
        if both:
            g.node("dw", "layer_norm_wgrad", ["dy", "x"], shared=[(y, 0), (y, 1)], eps=eps)
    return g


def norm_reference(x, gamma, beta, dy, eps):
    """In 64 bits: y, dx, dw, each with the largest error that the roundings of its formula allow, element by element.

    A sum over C channels is added up by threads that take up to k = max(16, C / 16) of them, then between threads: off by at most
    S u times the sum of the magnitudes, S = k + 22 (6 exchanges in a wavefront, at most 16 wavefronts). With A the mean magnitude and s the
    spread of a token: the mean is off by S u A, what is left after it by e = u |x - mean| + S u A, the variance by 2 e of its square
    root and S u in its own sum, so that r = 1 / spread is off by (S A / s + S / 2 + 5) u of itself, and xh by
    e_xh = u (S A / s (1 + |xh|) + (S / 2 + 7) |xh|). What follows are a handful of roundings and sums of the same kind."""
    f = lambda t: np.asarray(t, np.float64)  # noqa: E731
    eps = float(np.float32(eps))
    x, gamma, beta = f(x), f(gamma)[None, :, None, None], f(beta)[None, :, None, None]
    c = x.shape[1]
    S = max(16, c / 16) + 22
    centred = x - x.mean(1, keepdims=True)
    s = np.sqrt((centred ** 2).mean(1, keepdims=True) + eps)
    xh, A = centred / s, np.abs(x).mean(1, keepdims=True)
    e_xh = U * (S * A / s * (1 + np.abs(xh)) + (S / 2 + 7) * np.abs(xh))
    out = {"y": (xh * gamma + beta, np.abs(gamma) * e_xh + 4 * U * (np.abs(gamma * xh) + np.abs(beta)))}
    if dy is not None:
        dy = f(dy)
        dx, dg, db = layer_norm_vjp(x, gamma.ravel(), eps, dy)
        u = dy * gamma
        m1, m2 = u.mean(1, keepdims=True), (u * xh).mean(1, keepdims=True)
        off_r = U * (S * A / s + S / 2 + 5)
        off1 = (S + 2) * U * np.abs(u).mean(1, keepdims=True)
        off2 = (S + 3) * U * np.abs(u * xh).mean(1, keepdims=True) + (np.abs(u) * e_xh).mean(1, keepdims=True)
        inside = 3 * U * np.abs(u) + off1 + 3 * U * np.abs(m1) + np.abs(xh) * off2 + np.abs(m2) * e_xh + 4 * U * np.abs(xh * m2)
        out["dx"] = dx, (inside + (off_r + 3 * U) * (np.abs(u) + np.abs(m1) + np.abs(xh * m2))) / s
        # over P tokens: a thread walks at most ceil(P / 1024) blocks of four, within 4 ceil(P / 256) terms, then 8 + 16 + 32 sums of sums (fewer
        # where there are fewer tokens)
        P = x.size // c
        D = min(P, 4 * (P // 256 + 1) + 60) + 2
        off_g = (D * U * np.abs(dy * xh) + np.abs(dy) * e_xh).sum((0, 2, 3))
        out["dw"] = np.stack([dg, db]).reshape(2, c, 1, 1), np.stack([off_g, D * U * np.abs(dy).sum((0, 2, 3))]).reshape(2, c, 1, 1)
    return out


def within(got, reference, what):
    for name, (ref, bound) in reference.items():
        if name not in got:
            continue
        off = np.abs(np.asarray(got[name], np.float64) - ref)
        assert np.isfinite(got[name]).all() and (off <= bound).all(), (what, name, float(off.max()), float((off / np.maximum(bound, 1e-300)).max()))


def block_reference(name, *args):
    """An oracle formula with its result in 64 bits."""
    keep, ops._out = ops._out, lambda t: np.asarray(t, np.float64)
    try:
        return getattr(ops, name)(*args)
    finally:
        ops._out = keep
