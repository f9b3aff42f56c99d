"""Calls of the operators around a transformer block's attention that a user may make: tensors of more than 2^32 bytes, replays recorded into
the caller's own graph, a plan that hands buffers on, one attention's gradients for two dy."""
import numpy as np
import pytest
import torch

import workloads
from attention_util import Graph
from block_util import U, norm_reference, run, within
from oracle.ops import dropout_scale
from test_gpu_attention_calls import on_device
from test_gpu_biased_attention import biased_graph, check, inputs
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
DEV, F32 = "cuda:0", np.float32


def test_layer_norm_of_more_than_4_gib():
    """x, dy, y and dx of 4.4 GB each: the last image, which is all behind the first 2^32 bytes, against 64 bits, and both sums. 2-norms: mean
    and variance 22 u, three products, sums over 1.05 million tokens in parts: as in the test of tensors beyond the caches."""
    n, c, t = 3, 1023, 350001
    g = torch.Generator(DEV).manual_seed(1)
    x, dy = (torch.randn(n, c, 1, t, generator=g, device=DEV) for _ in range(2))
    assert x[:2].numel() * 4 < 1 << 32 < x.numel() * 4
    gamma, beta = np.linspace(0.5, 1.5, c).astype(F32), np.linspace(-1, 1, c).astype(F32)
    ops = [("y", "layer_norm", ["x"], x.shape, dict(eps=1e-5), [gamma, beta], []),
           ("dx", "layer_norm_dgrad", ["dy", "x"], x.shape, dict(eps=1e-5), [], [("y", 0), ("y", 1)]),
           ("dw", "layer_norm_wgrad", ["dy", "x"], (2, c, 1, 1), dict(eps=1e-5), [], [("y", 0), ("y", 1)])]
    w, ids = on_device(dict(x=x, dy=dy), ops)
    r = GraphRunner(w, DEV)
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        gm, bt = (torch.from_numpy(v).to(DEV).double()[:, None] for v in (gamma, beta))
        sums = torch.zeros(2, c, dtype=torch.float64, device=DEV)
        for i in range(n):
            for first in range(0, t, 50000):
                xs, gs = (v[i, :, 0, first:first + 50000].double() for v in (x, dy))
                rs = (xs.var(0, unbiased=False) + 1e-5).rsqrt()
                xh = (xs - xs.mean(0)) * rs
                sums += torch.stack([(gs * xh).sum(1), gs.sum(1)])
                if i == n - 1:
                    u = gs * gm
                    dx = rs * (u - u.mean(0) - xh * (u * xh).mean(0))
                    for name, ref in (("y", gm * xh + bt), ("dx", dx)):
                        off = float((r.tensor(ids[name])[i, :, 0, first:first + 50000].double() - ref).norm() / ref.norm())
                        assert off <= 40 * U, (name, first, off / U)
        off = float((r.tensor(ids["dw"]).view(2, c).double() - sums).norm() / sums.norm())
        assert off <= 40 * U, off / U
    finally:
        r.close()


@pytest.mark.parametrize("tq", [1, 150])
def test_biased_attention_of_more_than_4_gib(tq):
    """Keys and values of 4.3 GB each: the last tokens of a long sequence, with gradients, dbias too. Every head against 64 bits; the
    roundings per term as in test_memory_of_more_than_4_gib, the bias adds one of a score. The bias's gradient element by
    element as in test_gpu_biased_attention.check: a dP is a sum of d products, off by d U of their magnitudes' sum (not of its own, which may be
    anything down to zero: a bound by |dP| was 1.7 times too small at one element), the same for dot; a weight is off by 2 e, e = U ((d + 10) S +
    6 |bias|) with S the largest sum of a score's magnitudes; sums over 2^13 keys of a block's run."""
    heads, d, tk, reach = 4, 128, (1 << 21) + 37, 128
    g = torch.Generator(DEV).manual_seed(tq)
    q, dy = (torch.randn(1, heads * d, 1, tq, generator=g, device=DEV) for _ in range(2))
    k, v = (torch.randn(1, heads * d, 1, tk, generator=g, device=DEV) for _ in range(2))
    bias = torch.randn(1, heads, 1, 2 * reach + 1, generator=g, device=DEV)
    bias[..., reach + 1:] = -np.inf
    how = dict(heads=heads, kv_heads=heads, scale=d ** -0.5, bias="last")
    read = ["dy", "rows", "q", "k", "v", "bias"]
    ops = [("y", "attention", ["q", "k", "v", "bias"], q.shape, how, [], []), ("rows", "attention_rows", ["dy", "y"], (1, 3 * heads, 1, tq), dict(heads=heads), [], [])]
    ops += [(name, "attention_" + name, read, (q if name == "dq" else k).shape, how, [], []) for name in ("dq", "dk", "dv")]
    ops += [("db", "attention_dbias", read, bias.shape, how, [], [])]
    w, ids = on_device(dict(q=q, k=k, v=v, dy=dy, bias=bias), ops)
    r = GraphRunner(w, DEV)
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        got = {name: r.tensor(ids[name]).view(heads, d, -1) for name in ("y", "dq", "dk", "dv")}
        away = torch.arange(tk, device=DEV)[None, :] - (torch.arange(tq, device=DEV)[:, None] + tk - tq)
        away = away.clamp(-reach, reach) + reach
        far = tk - tq - reach                                   # of every query

        def along(t):
            sums = torch.zeros(2 * reach + 1, dtype=torch.float64, device=DEV)
            sums[0] = t[:, :far].sum()
            return sums.scatter_add_(0, away[:, far:].reshape(-1), t[:, far:].reshape(-1))

        for h in range(heads):
            qh, kh, vh, gh = (t.view(heads, d, -1)[h].double() for t in (q, k, v, dy))
            s = (qh.t() @ kh) * float(F32(d ** -0.5)) + bias[0, h, 0].double()[away]
            p = torch.softmax(s, 1)
            del s
            y = vh @ p.t()
            dp = gh.t() @ vh
            dot = (gh * y).sum(0)[:, None]
            ds = p * (dp - dot)
            ref = {"y": y, "dq": (kh @ ds.t()) * d ** -0.5, "dk": (qh @ ds) * d ** -0.5, "dv": gh @ p}
            may = 4 * U * 180 * 2
            for name, t in ref.items():
                off = float((got[name][h].double() - t).norm() / t.norm())
                assert off <= may, (name, h, off / may)
            db = along(ds)
            del ds
            del dp
            S = max(float((qh.abs().t() @ kh[:, i:i + 65536].abs()).max()) for i in range(0, tk, 65536)) * d ** -0.5
            e = U * ((d + 10) * S + 6 * float(bias[torch.isfinite(bias)].abs().max()))
            t = gh.abs().t() @ vh.abs()
            t = p * (t + (p * t).sum(1, keepdim=True))
            mag = along(t)
            off = (r.tensor(ids["db"])[0, h, 0].double() - db).abs()
            bound = (2 * e + (2 * d + 16) * U + (2 ** 13 / 32 + 120) * U) * mag
            assert bool((off <= bound).all()), (h, float((off / bound.clamp_min(1e-300)).max()))
            del qh, kh, vh, gh, p, y, t, dot, ref, db, mag
    finally:
        r.close()


def test_static_replay_of_norm_and_dropout_in_a_graph_of_the_callers():
    """ng_replay_static under capture, replayed on new inputs and new seeds between eager work and waits; two such graphs in turn."""
    stream = torch.cuda.Stream(DEV)
    runners = []
    try:
        for c, t in ((40, 90), (96, 50)):
            rng = np.random.default_rng(c)
            gamma, beta = (rng.standard_normal(c).astype(F32) for _ in range(2))
            g = Graph()
            g.given("x", np.zeros((2, c, 1, t), F32))
            g.given("seed", np.zeros((1, 1, 1, 2), F32))
            g.node("n", "layer_norm", ["x"], (2, c, 1, t), [gamma, beta], eps=1e-5)
            g.node("y", "dropout", ["n", "seed", "x"], (2, c, 1, t), rate=0.25, site=3)
            r = GraphRunner(g.workload(), DEV)
            runners.append(r)
            r.prepare(plan_trials=1, origin_stream=stream.cuda_stream)
            B.ng_replay_static(r.g)
            r.sync()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                B.ng_replay_static(r.g)
            r.own = (g, graph, gamma, beta, rng)
        for turn in range(4):
            for r in runners:
                g, graph, gamma, beta, rng = r.own
                x = rng.standard_normal((2, gamma.size, 1, r.tensor(g.names["y"]).shape[3])).astype(F32)
                seed = np.array([turn, 7 * turn + 1], F32).reshape(1, 1, 1, 2)
                r.set_input(x, g.names["x"]), r.set_input(seed, g.names["seed"])
                for name in ("n", "y"):
                    r.tensor(g.names[name]).fill_(float("nan"))
                torch.cuda.synchronize(DEV)
                with torch.cuda.stream(stream):
                    graph.replay()
                torch.cuda.synchronize(DEV)
                got = {name: r.output(g.names[name]) for name in ("n", "y")}
                ref = norm_reference(x, gamma, beta, None, 1e-5)["y"]
                within(got, {"n": ref}, turn)
                kept = dropout_scale(x.shape, seed, 0.25, 3) > 0
                y = x.astype(np.float64) + np.where(kept, got["n"].astype(np.float64) / 0.75, 0)
                assert (np.abs(got["y"] - y) <= 3 * U * (np.abs(x) + np.abs(got["n"]) / 0.75)).all(), turn
                r.replay(B.NG_MODE_GRAPH_SINGLE)
                assert all(np.array_equal(r.output(g.names[name]), got[name]) for name in got), turn
    finally:
        for r in runners:
            r.close()


def test_a_training_step_on_a_plan_that_hands_buffers_on():
    """The updated weights and the output of a block's training step, with every buffer of its own and with reuse."""
    w = workloads.transformer_block(batch=2, tokens=70, d=16, layers=1, max_distance=20, buckets=8)
    out = w.outputs[0]
    dy = np.random.default_rng(4).standard_normal(w.nodes[out].shape).astype(F32)
    places = [(v, j) for v, nd in enumerate(w.nodes) for j in range(len(nd.weights))]
    results = []
    for reuse, mode in ((0, B.NG_MODE_GRAPH_SINGLE), (1, B.NG_MODE_GRAPH_SINGLE), (1, B.NG_MODE_GRAPH_MULTI), (1, B.NG_MODE_EAGER_MULTI)):
        tw = workloads.training_graph(w, 1e-3, {out: dy})
        r = GraphRunner(tw, DEV)
        try:
            B.ng_set_memory_reuse(r.g, reuse)
            r.prepare(plan_trials=1)
            r.arena.fill_(0xFF)
            for v, t in tw.inputs.items():
                r.set_input(t, v)
            for v, j in places:                                 # (ng_capture's own replays have moved them)
                r.set_weight(v, j, w.nodes[v].weights[j])
            r.replay(mode)
            r.sync()
            results.append([r.weight(v, j) for v, j in places])
        finally:
            r.close()
    for other in results[1:]:
        for (v, j), a, b in zip(places, results[0], other):
            keep = w.nodes[v].weights[j]
            moved = np.abs(a.astype(np.float64) - keep).max()
            assert np.isfinite(b).all() and np.abs(a - b).max() <= 1e-3 * moved + 4 * U * np.abs(keep).max(), (v, w.nodes[v].op, j)
    assert all(np.array_equal(a, b) for a, b in zip(results[0], results[1])), "reuse changes a result"


@pytest.mark.parametrize("sizes", [(2, 4, 2, 64, 40, 90, "first"), (2, 8, 4, 64, 150, 333, "last"), (2, 8, 4, 128, 150, 333, "first")], ids=str)
def test_gradients_for_two_dy_of_one_biased_attention(sizes):
    """Two parts of a network that read the same attention, each with gradients of its own."""
    n, heads, kv, d, tq, tk, at = sizes
    q, k, v, dy, ln, bias = inputs(5, n, heads, kv, d, tq, tk, "ragged", 20, "back")
    dy2 = np.random.default_rng(6).standard_normal(dy.shape).astype(F32)
    g = biased_graph(q, k, v, dy, ln, bias, heads, kv, d ** -0.5, at)
    how = dict(heads=heads, kv_heads=kv, scale=d ** -0.5, bias=at)
    g.given("dy2", dy2)
    g.node("rows2", "attention_rows", ["dy2", "y"], heads=heads)
    first = g.nodes[g.names["dq"]].preds
    names = {i: name for name, i in g.names.items()}
    read = ["dy2", "rows2"] + [names[p] for p in first[2:]]
    for name, op in (("db2", "attention_dbias"), ("dq2", "attention_dq"), ("dv2", "attention_dv")):
        g.node(name, op, read, **how)
    for mode, t in run(g, (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_MULTI)).items():
        check(t, q, k, v, dy, ln, bias, heads, kv, d ** -0.5, at, (sizes, mode))
        check({"y": t["y"], "rows": t["rows2"], "db": t["db2"], "dq": t["dq2"], "dv": t["dv2"]}, q, k, v, dy2, ln, bias, heads, kv, d ** -0.5, at, (sizes, mode, 2))
