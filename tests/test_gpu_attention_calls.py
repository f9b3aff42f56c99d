"""Calls of the attention operators that a user may make: tensors of more than 2^32 bytes, replays recorded into the caller's own graph, one
attention's gradients for two dy, one tensor in several places."""
import numpy as np
import pytest
import torch

import workloads
from attention_bounds import MARGIN, U, check, reference_and_rss, excess
from attention_util import Graph, attention_graph
from test_gpu_attention import DEV, attention_inputs, run
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu


def on_device(inputs, ops):
    """A graph whose inputs are device tensors by name; ops: (name, op, preds, shape, params, weights, shared)."""
    nodes, values, ids = [], {}, {}
    for name, t in inputs.items():
        ids[name], values[len(nodes)] = len(nodes), t
        nodes.append(workloads.Node("input", [], dict(zip("nchw", t.shape)), [], tuple(t.shape)))
    for name, op, preds, shape, params, weights, shared in ops:
        ids[name] = len(nodes)
        nodes.append(workloads.Node(op, [ids[p] for p in preds], params, list(weights), tuple(shape), 1.0, [(ids[n], j) for n, j in shared]))
    w = workloads.Workload("calls", nodes, values[0], [ids[o[0]] for o in ops], inputs=values)
    return w, ids


@pytest.mark.parametrize("tq", [1, 48])
def test_memory_of_more_than_4_gib(tq):
    """Keys and values of 4.3 GB each, a head's 1.07 GB: one token, and a prompt through LDS, with gradients. Every head against 64 bits."""
    heads, d, tk = 4, 128, (1 << 21) + 37
    g = torch.Generator(DEV).manual_seed(tq)
    q, dy = (torch.randn(1, heads * d, 1, tq, generator=g, device=DEV) for _ in range(2))
    k, v = (torch.randn(1, heads * d, 1, tk, generator=g, device=DEV) for _ in range(2))
    assert k.numel() * 4 > 1 << 32
    k[..., 3::7] *= 1.5
    how = dict(heads=heads, kv_heads=heads, scale=d ** -0.5)
    ops = [("y", "attention", ["q", "k", "v"], q.shape, how, [], []), ("rows", "attention_rows", ["dy", "y"], (1, 3 * heads, 1, tq), dict(heads=heads), [], [])]
    ops += [(name, "attention_" + name, ["dy", "rows", "q", "k", "v"], (q if name == "dq" else k).shape, how, [], []) for name in ("dq", "dk", "dv")]
    w, ids = on_device(dict(q=q, k=k, v=v, dy=dy), ops)
    r = GraphRunner(w, DEV)
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        got = {name: r.tensor(ids[name]).view(heads, d, -1) for name in ("y", "dq", "dk", "dv")}
        for h in range(heads):
            qh, kh, vh, gh = (t.view(heads, d, -1)[h].double() for t in (q, k, v, dy))
            s = (qh.t() @ kh) * float(np.float32(d ** -0.5))
            p = torch.softmax(s, 1)
            y = vh @ p.t()
            ds = p * (gh.t() @ vh - (gh * y).sum(0)[:, None])
            ref = {"y": y, "dq": (kh @ ds.t()) * d ** -0.5, "dk": (qh @ ds) * d ** -0.5, "dv": gh @ p}
            # per term (attention_bounds.py): scores of up to 9, sums of 128 and of 2^21 terms, which the splits cut into blocks of
            # 2^13 at most: sqrt(128) 2 + 45 + sqrt(128) + sqrt(2^13) + 16; relative to the 2-norm of the terms, which for y and dq of
            # even weights is the result's own but for a factor of 2
            may = MARGIN * U * 175 * 2
            for name, t in ref.items():
                off = float((got[name][h].double() - t).norm() / t.norm())
                assert off <= may, (name, h, off / may)
            del qh, kh, vh, gh, s, p, y, ds, ref, t
    finally:
        r.close()


def test_norm_and_rotation_of_more_than_4_gib():
    """x and y of 4.3 GB each, and both gradients: the last image, which is all behind the first 2^32 bytes, against 64 bits."""
    n, heads, d, tokens = 3, 40, 128, 70001
    g = torch.Generator(DEV).manual_seed(1)
    x, dy = (torch.randn(n, heads * d, 1, tokens, generator=g, device=DEV) for _ in range(2))
    assert x[:2].numel() * 4 < 1 << 32 < x.numel() * 4
    pos = torch.arange(tokens, device=DEV, dtype=torch.float32).view(1, 1, 1, tokens)
    freq, gamma = workloads.rope_frequencies(d), np.linspace(0.5, 1.5, d).astype(np.float32)
    how = dict(heads=heads, rot=d, interleaved=0, eps=1e-6, factor=1.0)
    ops = [("y", "head_rope", ["x", "pos"], x.shape, how, [freq, gamma], []),
           ("dx", "head_rope_dgrad", ["dy", "x", "pos"], x.shape, how, [], [("y", 0), ("y", 1)]),
           ("dgamma", "head_rope_wgrad", ["dy", "x", "pos"], (1, d, 1, 1), how, [], [("y", 0), ("y", 1)])]
    w, ids = on_device(dict(x=x, pos=pos, dy=dy), ops)
    r = GraphRunner(w, DEV)
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        angle = pos.view(1, tokens).double() * torch.from_numpy(freq).to(DEV).double()[:, None]
        cos, sin, half = torch.cos(angle), torch.sin(angle), d // 2
        gm = torch.from_numpy(gamma).to(DEV).double()[:, None]
        dgamma = torch.zeros(d, dtype=torch.float64, device=DEV)
        for i in range(n):
            for h in range(heads):
                xh, gh = (t[i].view(heads, d, tokens)[h].double() for t in (x, dy))
                rms = (xh.square().mean(0) + 1e-6).sqrt()
                u = xh / rms * gm
                du = torch.cat([gh[:half] * cos + gh[half:] * sin, gh[half:] * cos - gh[:half] * sin])
                dgamma += (du * xh / rms).sum(1)
                if i < n - 1 or h % 13:
                    continue
                y = torch.cat([u[:half] * cos - u[half:] * sin, u[:half] * sin + u[half:] * cos])
                gu, xn = du * gm, xh / rms
                dx = (gu - xn * (gu * xn).mean(0)) / rms
                for name, t in (("y", y), ("dx", dx)):           # a sum of 128 squares, a handful of roundings
                    off = float((r.tensor(ids[name])[i].view(heads, d, tokens)[h].double() - t).norm() / t.norm())
                    assert off <= 2 * (np.sqrt(d) + 16) * U, (name, i, h, off / U)
        # terms of order one: sums of up to 2^14 of them in a thread, then of 512 rows; random roundings
        got = r.tensor(ids["dgamma"]).view(-1).double()
        assert float((got - dgamma).abs().max()) <= 4 * np.sqrt(n * heads * tokens) * (np.sqrt(1 << 14) + 16) * U
    finally:
        r.close()


def test_static_replay_recorded_into_a_graph_of_the_callers():
    """ng_replay_static under capture: the caller's graph is replayed several times, on new inputs, between eager work and waits."""
    stream = torch.cuda.Stream(DEV)
    q, k, v, dy, ln = attention_inputs(3, 2, 4, 2, 100, 20, 300, "ragged")      # kernels that the resident build has
    g = attention_graph(q, k, v, dy, ln, 4, 2, 0.2)
    r = GraphRunner(g.workload(), DEV)
    try:
        r.prepare(plan_trials=1, origin_stream=stream.cuda_stream)
        B.ng_replay_static(r.g)
        r.sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            B.ng_replay_static(r.g)
        for turn in range(4):
            q, k, v, dy, ln = attention_inputs(100 + turn, 2, 4, 2, 100, 20, 300, "ragged")
            for name, t in (("q", q), ("k", k), ("v", v), ("dy", dy), ("lengths", ln)):
                r.set_input(t, g.names[name])
            for name in ("y", "dq", "dk", "dv"):
                r.tensor(g.names[name]).fill_(float("nan"))
            torch.cuda.synchronize(DEV)
            with torch.cuda.stream(stream):
                graph.replay()
            torch.cuda.synchronize(DEV)
            got = {name: r.output(g.names[name]) for name in ("y", "dq", "dk", "dv")}
            check(got, q, np.nan_to_num(k), np.where(np.isfinite(v), v, 0), dy, ln, 4, 2, 0.2, turn)
            r.replay(B.NG_MODE_GRAPH_SINGLE)
            assert all(np.array_equal(r.output(g.names[name]), got[name]) for name in got), turn
    finally:
        r.close()


@pytest.mark.parametrize("sizes", [(2, 4, 2, 64, 40, 90), (2, 8, 4, 64, 150, 333), (2, 8, 4, 128, 150, 333)], ids=str)
def test_gradients_for_two_dy_of_one_attention(sizes):
    """Two heads of a network that read the same attention, each with gradients of its own; the second without dq."""
    n, heads, kv_heads, d, tq, tk = sizes
    q, k, v, dy, ln = attention_inputs(5, n, heads, kv_heads, d, tq, tk, "ragged")
    dy2 = np.random.default_rng(6).standard_normal(dy.shape).astype(np.float32)
    g = attention_graph(q, k, v, dy, ln, heads, kv_heads, d ** -0.5)
    g.given("dy2", dy2)
    g.node("rows2", "attention_rows", ["dy2", "y"], heads=heads)
    for name in ("dv", "dk"):
        g.node(name + "2", "attention_" + name, ["dy2", "rows2", "q", "k", "v", "lengths"], heads=heads, kv_heads=kv_heads, scale=d ** -0.5)
    got = run(g, (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_MULTI))
    k, v = np.nan_to_num(k), np.where(np.isfinite(v), v, 0)
    for mode, t in got.items():
        check(t, q, k, v, dy, ln, heads, kv_heads, d ** -0.5, (sizes, mode))
        ref, rss = reference_and_rss(q, k, v, dy2, ln, heads, kv_heads, d ** -0.5)
        for name in ("dk", "dv"):
            assert excess({name: t[name + "2"]}, {name: ref[name]}, {name: rss[name]})[name] <= 1, (sizes, mode, name)


@pytest.mark.parametrize("d,tokens", [(64, 30), (64, 300), (128, 300)])
def test_one_tensor_as_queries_keys_values_and_dy(d, tokens):
    rng = np.random.default_rng(d + tokens)
    x = rng.standard_normal((2, 4 * d, 1, tokens)).astype(np.float32)
    g, how = Graph(), dict(heads=4, kv_heads=4, scale=d ** -0.5)
    g.given("x", x)
    g.node("y", "attention", ["x", "x", "x"], x.shape, **how)
    g.node("rows", "attention_rows", ["x", "y"], heads=4)
    for name in ("dq", "dk", "dv"):
        g.node(name, "attention_" + name, ["x", "rows", "x", "x", "x"], **how)
    for mode, t in run(g, (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_DEVICE_RESIDENT)).items():
        check(t, x, x, x, x, None, 4, 4, d ** -0.5, (d, tokens, mode))
