"""Attention operators on the GPU against the oracle's formulas in 64 bits: norm and rotation of heads, attention to another
sequence's states, and their gradients, in every replay mode.

Tolerances. u = 2^-24, half a step of fp32. A sum of n rounded products is off by at most about n u times the sum of the magnitudes,
and by about sqrt(n) u times their root mean square; the tests bound the largest error by the former and the 2-norm by the latter, with
a margin of four for what follows the sum (exp2, a division, a second product).
  scores     |error| <= (d + 4) u S, S = largest scale sum |q| |k| of a pair: the relative error of every softmax weight is twice that
  y          |error| <= (2 (d + 4) S + Tk + 8) u max|v|; 2-norm: (sqrt(d) + sqrt(min(Tk, 256)) + 8) u, times 4
  gradients  the same weights, then sums of up to n = max(d, Tk, G Tq) terms: 2-norm (2 sqrt(d) + 2 sqrt(min(n, 1024)) + 16) u, times 4,
             relative to the 2-norm that the sums of magnitudes have (the terms of dS cancel)
  rotation   angles to u of half a turn: 4 u; norm and rotation a handful of roundings: (sqrt(d) + 16) u of the largest value
"""
import numpy as np
import pytest

from attention_util import attention_graph, attention_reference, rope_graph, rope_reference
from paper_2012_02732_amd import GraphRunner, binding as B
from workloads import rope_frequencies

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
MODES = (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_SINGLE, B.NG_MODE_EAGER_MULTI, B.NG_MODE_DEVICE_RESIDENT)


def run(g, modes=(B.NG_MODE_GRAPH_SINGLE,), **prepare):
    """{mode: {name: tensor}}; a mode without a plan is left out."""
    r = GraphRunner(g.workload(), DEV)
    try:
        r.prepare(plan_trials=1, **prepare)
        got = {}
        for mode in modes:
            r.arena.fill_(0xFF)                                 # a tensor that is not written stays NaN
            for v, t in g.inputs.items():
                r.set_input(t, v)
            try:
                r.replay(mode)
            except B.NgError as e:
                assert mode in (B.NG_MODE_DEVICE_RESIDENT, B.NG_MODE_GRAPH_MULTI) and e.code == B.NG_ESTATE, (mode, e)
                continue
            r.sync()
            got[mode] = {name: r.output(v) for name, v in g.names.items() if v not in g.inputs}
        return got
    finally:
        r.close()


def norm_off(got, ref):
    return float(np.linalg.norm(np.asarray(got, np.float64) - ref) / max(np.linalg.norm(ref), 1e-300))


def lengths_of(kind, n, tk):
    if kind is None:
        return None
    few = {"ragged": [tk, tk // 2, 0, tk - 1, 1], "odd": [tk - 0.5, float("nan"), -3.0, 1e9, 0.25]}[kind]
    return np.array([few[i % len(few)] for i in range(n)], np.float32).reshape(n, 1, 1, 1)


def attention_inputs(seed, n, heads, kv_heads, d, tq, tk, lengths, dy_scale=1.0):
    rng = np.random.default_rng(seed)
    q, dy = (rng.standard_normal((n, heads * d, 1, tq)).astype(np.float32) for _ in range(2))
    k, v = (rng.standard_normal((n, kv_heads * d, 1, tk)).astype(np.float32) for _ in range(2))
    ln = lengths_of(lengths, n, tk)
    if ln is not None:                                          # whatever lies behind the keys that count must not matter
        for b in range(n):
            m = int(min(max(np.ceil(np.nan_to_num(ln[b, 0, 0, 0], nan=0.0)), 0), tk))
            k[b, :, :, m:], v[b, :, :, m:] = np.nan, np.inf
    return q, k, v, (dy * dy_scale).astype(np.float32), ln


def check_attention(got, q, k, v, dy, ln, heads, kv_heads, scale, what):
    n, d, tq, tk = q.shape[0], q.shape[1] // heads, q.shape[3], k.shape[3]
    clean = [np.where(np.isfinite(t), t, 0).astype(np.float64) for t in (k, v)]
    ref = attention_reference(q, clean[0], clean[1], dy, ln, heads, kv_heads, scale)
    group = heads // kv_heads
    qa, ka = np.abs(q.reshape(n, kv_heads, group, d, tq)).astype(np.float64), np.abs(clean[0].reshape(n, kv_heads, 1, d, tk))
    top = abs(scale) * (qa.transpose(0, 1, 2, 4, 3) @ ka).max()
    assert np.isfinite(got["y"]).all(), what
    bound = (2 * (d + 4) * top + tk + 8) * U * np.abs(clean[1]).max()
    assert np.abs(got["y"] - ref["y"]).max() <= bound, (what, "y", np.abs(got["y"] - ref["y"]).max(), bound)
    assert norm_off(got["y"], ref["y"]) <= 4 * (np.sqrt(d) * max(1.0, abs(scale) * d ** 0.5) + np.sqrt(min(tk, 256)) + 8) * U, (what, "y", norm_off(got["y"], ref["y"]))
    if ln is not None:
        for b in range(n):
            m = int(min(max(np.ceil(np.nan_to_num(ln[b, 0, 0, 0], nan=0.0)), 0), tk))
            if m == 0:
                assert not got["y"][b].any(), (what, b)
            if "dk" in got:
                assert not got["dk"][b, :, :, m:].any() and not got["dv"][b, :, :, m:].any(), (what, b)
    if "dq" in got:
        # magnitudes: what the terms of each sum add up to without cancellation
        w = {"dv": attention_reference(q, clean[0], clean[1], np.abs(dy), ln, heads, kv_heads, scale)["dv"]}
        largest = max(d, tk, group * tq)
        tol = 4 * (2 * np.sqrt(d) * max(1.0, abs(scale) * d ** 0.5) + 2 * np.sqrt(min(largest, 1024)) + 16) * U
        gy = np.linalg.norm(dy.astype(np.float64).reshape(n, heads, d, tq), axis=2)          # |dy| of each query
        spread = np.sqrt(d) * np.abs(clean[1]).max()
        for name, other in (("dq", clean[0]), ("dk", q.astype(np.float64))):
            # dS <= p |dy| |v|, summed with p = 1 over keys: |dq| <= scale |dy| |v| |k|; dk over queries likewise
            scale_of = abs(scale) * spread * np.abs(other).max() * np.sqrt((gy ** 2).sum())
            off = np.linalg.norm(got[name] - ref[name])
            assert np.isfinite(got[name]).all() and off <= tol * max(scale_of, 1e-300), (what, name, off, tol * scale_of)
            # one key has p = 1 and dS = dp - <dy, y> = 0 whatever the inputs: nothing to be relative to
            assert tk == 1 or norm_off(got[name], ref[name]) <= 100 * tol, (what, name, norm_off(got[name], ref[name]))
        assert np.linalg.norm(got["dv"] - ref["dv"]) <= tol * np.linalg.norm(w["dv"]), (what, "dv", norm_off(got["dv"], ref["dv"]))


ATTENTION = [                   # n, heads, kv_heads, d, Tq, Tk, lengths
    (1, 1, 1, 1, 1, 1, None),
    (2, 2, 1, 8, 1, 3, "odd"),
    (5, 2, 2, 16, 3, 5, "odd"),
    (2, 4, 2, 40, 17, 77, None),
    (5, 8, 1, 64, 1, 200, "ragged"),
    (1, 3, 3, 7, 5, 129, None),
    (3, 4, 4, 64, 33, 64, "ragged"),
    (1, 2, 2, 128, 130, 65, None),
    (5, 4, 2, 128, 19, 63, "odd"),
    (2, 16, 2, 100, 1, 1030, "ragged"),
    (1, 2, 1, 65, 2, 4099, None),
    (1, 1, 1, 33, 700, 1, None),
    (2, 6, 2, 64, 257, 333, "ragged"),
    (1, 4, 4, 128, 300, 520, None),
    (2, 2, 2, 128, 129, 1, None),
    (3, 3, 1, 48, 43, 97, "ragged"),
    (1, 1, 1, 128, 40, 2050, None),
    (4, 2, 2, 64, 64, 3000, "ragged"),
    (1, 8, 2, 96, 33, 31, None),
]


@pytest.mark.parametrize("case", ATTENTION, ids=str)
def test_attention_and_gradients(case):
    n, heads, kv_heads, d, tq, tk, kind = case
    q, k, v, dy, ln = attention_inputs(tq * 1000 + tk, n, heads, kv_heads, d, tq, tk, kind)
    scale = d ** -0.5
    g = attention_graph(q, k, v, dy, ln, heads, kv_heads, scale)
    got = run(g, MODES)
    first = got[B.NG_MODE_GRAPH_SINGLE]
    check_attention(first, q, k, v, dy, ln, heads, kv_heads, scale, case)
    for mode, tensors in got.items():                           # the same kernels and order of sums: bit for bit
        for name in tensors:
            assert np.array_equal(tensors[name], first[name]), (case, mode, name)


@pytest.mark.parametrize("magnitude", [1e-20, 1e-6, 1e6, 1e15])
def test_attention_of_values_far_from_one(magnitude):
    """v, and with it dv's partner dy, of any magnitude; scores stay of order one."""
    q, k, v, dy, ln = attention_inputs(5, 2, 4, 2, 64, 70, 90, None, dy_scale=1.0)
    v, dy = (v * np.float32(magnitude)).astype(np.float32), (dy / np.float32(magnitude)).astype(np.float32)
    g = attention_graph(q, k, v, dy, ln, 4, 2, 0.125)
    check_attention(run(g)[B.NG_MODE_GRAPH_SINGLE], q, k, v, dy, ln, 4, 2, 0.125, magnitude)


@pytest.mark.parametrize("magnitude", [1e-12, 1e12])
def test_attention_of_queries_and_keys_far_from_one(magnitude):
    """q small and k large or the other way round: the scores are of order one."""
    q, k, v, dy, ln = attention_inputs(6, 1, 2, 2, 48, 40, 50, None)
    q, k = (q * np.float32(magnitude)).astype(np.float32), (k / np.float32(magnitude)).astype(np.float32)
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.2)
    got = run(g)[B.NG_MODE_GRAPH_SINGLE]
    ref = attention_reference(q, k, v, dy, ln, 2, 2, 0.2)
    for name in ("y", "dq", "dk", "dv"):
        assert norm_off(got[name], ref[name]) <= 400 * U, (name, norm_off(got[name], ref[name]))


def test_attention_with_channels_and_tokens_of_very_different_size():
    """A value among small ones is 2^20 times as large: the small ones keep what fp32 sums of their own would have of them."""
    q, k, v, dy, ln = attention_inputs(7, 1, 2, 2, 64, 96, 200, None)
    v[:, :, :, 50] *= 2.0 ** 20
    k[:, :, :, 51] *= 2.0 ** -20
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.125)
    check_attention(run(g)[B.NG_MODE_GRAPH_SINGLE], q, k, v, dy, ln, 2, 2, 0.125, "spread")


def test_attention_sharp_softmax():
    """Scores of hundreds: the largest key takes nearly everything, weights of the others vanish, nothing overflows."""
    q, k, v, dy, ln = attention_inputs(8, 2, 2, 2, 32, 50, 300, None)
    g = attention_graph(q, k, v, dy, ln, 2, 2, 20.0)
    got = run(g)[B.NG_MODE_GRAPH_SINGLE]
    ref = attention_reference(q, k, v, dy, ln, 2, 2, 20.0)
    # scores of up to S = 20 sum |q| |k| are off by sqrt(d) u S, and that is the relative error of the weights
    top = 20.0 * np.abs(q).max() * np.abs(k).max() * 32
    assert np.isfinite(got["y"]).all() and norm_off(got["y"], ref["y"]) <= 2 * 6 * U * top


ROPE = [                        # n, heads, d, rot, T, interleaved, norm, positions of each image
    (1, 1, 2, 2, 1, 0, True, False),
    (3, 4, 64, 64, 1, 0, True, True),
    (2, 5, 128, 128, 1, 1, True, True),
    (2, 3, 96, 24, 5, 1, False, True),
    (1, 2, 7, 4, 15, 0, True, False),
    (2, 3, 40, 20, 16, 1, True, True),
    (3, 8, 64, 64, 67, 0, True, False),
    (2, 2, 129, 128, 70, 1, True, True),
    (1, 3, 256, 200, 130, 0, True, True),
    (2, 2, 255, 2, 3, 0, True, False),
    (1, 2, 96, 96, 509, 0, False, True),
    (40, 2, 32, 32, 333, 1, True, True),
    (2, 1, 16, 16, 4096, 0, True, False),
]


@pytest.mark.parametrize("case", ROPE, ids=str)
def test_head_rope_and_gradients(case):
    n, heads, d, rot, tokens, interleaved, norm, each = case
    rng = np.random.default_rng(tokens)
    x, dy = (rng.standard_normal((n, heads * d, 1, tokens)).astype(np.float32) * 3 for _ in range(2))
    pos = rng.integers(0, 1 << 20, (n if each else 1, 1, 1, tokens)).astype(np.float32)
    freq = rope_frequencies(rot, scaling="ntk", factor=4.0)
    gamma = rng.uniform(0.5, 1.5, d).astype(np.float32) if norm else None
    args = (x, pos, freq, gamma, dy, heads, interleaved, 1e-6, 1.25)
    got, ref = run(rope_graph(*args), MODES), rope_reference(*args)
    first = got[B.NG_MODE_GRAPH_SINGLE]
    for name in ref:
        # sums of d squares (and of tokens x heads values for dgamma), then a handful of roundings
        count = d + (n * heads * tokens if name == "dgamma" else 0)
        tol = 2 * (np.sqrt(count) + 16) * U
        scale = np.abs(ref[name]).max() if name != "dgamma" else 3 * 1.25 * np.sqrt(n * heads * tokens)     # the sum's terms are of order 3.75
        off = np.abs(first[name] - ref[name]).max()
        assert off <= tol * scale, (case, name, off, tol * scale)
    for mode, tensors in got.items():
        for name in tensors:
            assert np.array_equal(tensors[name], first[name]), (case, mode, name)


def test_head_rope_far_and_odd_positions():
    """Negative, fractional and far positions; the angle comes from the exact product."""
    x = np.ones((1, 64, 1, 20), np.float32)
    pos = np.array([0.0, -1.0, 0.5, 1e6 + 1, 16777215.0] * 4, np.float32).reshape(1, 1, 1, 20)
    args = (x, pos, rope_frequencies(64), None, x, 1, 0, 0.0, 1.0)
    got, ref = run(rope_graph(*args))[B.NG_MODE_GRAPH_SINGLE], rope_reference(*args)
    for name in ref:
        assert np.abs(got[name] - ref[name]).max() <= 16 * U * 1.5


def test_zero_rows_and_eps():
    """A head of zeros: u = 0 whatever eps is; the gradient is gamma g / sqrt(eps)."""
    x = np.zeros((1, 8, 1, 16), np.float32)
    dy = np.random.default_rng(0).standard_normal(x.shape).astype(np.float32)
    args = (x, np.zeros((1, 1, 1, 16), np.float32), rope_frequencies(8), np.ones(8, np.float32), dy, 1, 0, 1e-6, 1.0)
    got, ref = run(rope_graph(*args))[B.NG_MODE_GRAPH_SINGLE], rope_reference(*args)
    assert not got["y"].any() and not got["dgamma"].any()
    assert np.abs(got["dx"] - ref["dx"]).max() <= 32 * U * np.abs(ref["dx"]).max()


# ---- together, as a network has them --------------------------------------------------------------------------------------

def _decoder_training(**sizes):
    import workloads
    w = workloads.decoder_block(**sizes)
    out = w.outputs[0]
    seed = np.random.default_rng(1).standard_normal(w.nodes[out].shape).astype(np.float32)
    return w, out, seed, workloads.training_graph(w, 0.01, {out: seed})


@pytest.mark.parametrize("sizes", [{}, dict(batch=3, heads=8, kv_heads=2, d=64, tokens=150, states=211)], ids=["small", "larger"])
def test_training_step_of_a_block_with_attention(sizes):
    """Forward pass, gradients and update of a decoder block as one graph, in every mode that has a plan for it: gradients against the
    oracle on the forward tensors that the GPU stored, updated weights against its update, and the weights as they were after capture."""
    from oracle.backward import sgd_step
    from oracle.forward import eval_node
    from test_gpu_training import oracle_backward_on, rel_err
    w, out, seed, tw = _decoder_training(**sizes)
    for mode in (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_MULTI, B.NG_MODE_AUTO):
        r = GraphRunner(tw, DEV)
        try:
            r.prepare(plan_trials=1)
            for v, nd in enumerate(w.nodes):
                for j, t in enumerate(nd.weights):
                    assert np.array_equal(r.weight(v, j), t), (mode, v, j)
            with pytest.raises(B.NgError) as e:                 # a graph that trains next to attention: no device-resident plan
                r.replay(B.NG_MODE_DEVICE_RESIDENT)
            assert e.value.code == B.NG_ESTATE
            r.arena.zero_()
            for v, t in tw.inputs.items():
                r.set_input(t, v)
            r.replay(mode)
            r.sync()
            values = {v: r.output(v) for v in range(len(w.nodes))}
            for v, nd in enumerate(w.nodes):
                if nd.op != "input":
                    assert rel_err(values[v], eval_node(nd, [values[u] for u in nd.preds])) <= 1e-4, (mode, v, nd.op)
            d_value, d_weight = oracle_backward_on(w, values, {out: seed})
            for v, node in tw.grad_of.items():
                assert rel_err(r.output(node), d_value[v]) <= 1e-4, (mode, v, w.nodes[v].op)
            for (v, j), (node, offset, numel) in tw.wgrad_of.items():
                grad = r.output(node).ravel()[offset:offset + numel]
                assert rel_err(grad, d_weight[v][j].ravel()) <= 1e-4, (mode, v, j, w.nodes[v].op)
                new = sgd_step([w.nodes[v].weights[j]], [grad.reshape(w.nodes[v].weights[j].shape)], tw.lr)[0]
                assert rel_err(r.weight(v, j), new) <= 1e-6, (mode, v, j)
        finally:
            r.close()


def test_replays_follow_their_inputs_and_each_other():
    """One captured graph, new inputs between replays, eager work of the program in between; then two graphs on one stream."""
    import torch
    graphs, streams = [], torch.cuda.Stream(DEV)
    for seed in (0, 1):
        q, k, v, dy, ln = attention_inputs(seed, 2, 4, 2, 32, 40, 300, "ragged")
        g = attention_graph(q, k, v, dy, ln, 4, 2, 0.2)
        r = GraphRunner(g.workload(), DEV)
        r.prepare(plan_trials=1, origin_stream=streams.cuda_stream)
        graphs.append((g, r))
    try:
        for turn in range(4):
            refs = []
            for i, (g, r) in enumerate(graphs):
                q, k, v, dy, ln = attention_inputs(10 * turn + i, 2, 4, 2, 32, 40, 300, "ragged")
                for name, t in (("q", q), ("k", k), ("v", v), ("dy", dy), ("lengths", ln)):
                    r.set_input(t, g.names[name])
                refs.append((q, k, v, dy, ln))
            for g, r in graphs:
                r.replay(B.NG_MODE_GRAPH_SINGLE)
            junk = torch.randn(1 << 20, device=DEV).sum().item()             # unrelated work on torch's own stream
            for (g, r), ref in zip(graphs, refs):
                got = {name: r.output(i) for name, i in g.names.items() if i not in g.inputs}
                check_attention(got, *ref, 4, 2, 0.2, (turn, junk))
    finally:
        for g, r in graphs:
            r.close()


@pytest.mark.parametrize("case", [(1, 1, 1, 64, 256, 256, None), (2, 8, 8, 64, 128, 77, "ragged"), (4, 8, 8, 128, 48, 512, "ragged"), (16, 16, 16, 64, 64, 64, "odd"),
                                  (8, 8, 8, 40, 256, 77, None), (4, 4, 4, 128, 128, 128, None)], ids=str)
def test_attention_on_both_sides_of_the_choice_of_kernels(case):
    n, heads, kv_heads, d, tq, tk, kind = case
    q, k, v, dy, ln = attention_inputs(tq + tk, n, heads, kv_heads, d, tq, tk, kind)
    g = attention_graph(q, k, v, dy, ln, heads, kv_heads, d ** -0.5)
    check_attention(run(g)[B.NG_MODE_GRAPH_SINGLE], q, k, v, dy, ln, heads, kv_heads, d ** -0.5, case)


@pytest.mark.parametrize("case", [(1, 4, 4, 64, 40, 5000, None), (1, 3, 3, 128, 47, 3100, "ragged"), (1, 16, 2, 96, 500, 93, None), (2, 8, 1, 48, 700, 60, "odd"),
                                  (9, 5, 5, 32, 130, 140, "ragged")], ids=str)
def test_attention_cut_into_many_splits(case):
    """Few columns against a long other side (32 splits at most), and so many columns that one or two are best."""
    n, heads, kv_heads, d, tq, tk, kind = case
    q, k, v, dy, ln = attention_inputs(tq + tk, n, heads, kv_heads, d, tq, tk, kind)
    g = attention_graph(q, k, v, dy, ln, heads, kv_heads, d ** -0.5)
    got = run(g)
    for mode, tensors in got.items():
        check_attention(tensors, q, k, v, dy, ln, heads, kv_heads, d ** -0.5, (case, mode))


@pytest.mark.parametrize("dy_size,v_size", [(1e-20, 1e-11), (1e-33, 1.0), (1e-3, 1e-30)])
def test_attention_gradients_of_small_products(dy_size, v_size):
    """<dy, v> far below one, but a normal number: 2^-100 and less."""
    q, k, v, dy, ln = attention_inputs(9, 2, 4, 2, 64, 200, 300, "ragged", dy_scale=dy_size)
    v = np.where(np.isfinite(v), v * np.float32(v_size), v).astype(np.float32)
    g = attention_graph(q, k, v, dy, ln, 4, 2, 0.125)
    got = run(g)[B.NG_MODE_GRAPH_SINGLE]
    ref = attention_reference(q, np.nan_to_num(k), np.where(np.isfinite(v), v, 0), dy, ln, 4, 2, 0.125)
    for name in ("y", "dq", "dk", "dv"):                        # sums of a few hundred terms that cancel: as in check_attention, 400 u
        assert norm_off(got[name], ref[name]) <= 400 * U, (name, norm_off(got[name], ref[name]))


@pytest.mark.parametrize("how", ["reuse", "no_fusion", "device_scope"])
def test_attention_under_other_plans(how):
    """Buffers handed on, one launch for each task, every hand-over through device scope: the same results."""
    q, k, v, dy, ln = attention_inputs(11, 3, 4, 2, 40, 50, 90, "ragged")
    g = attention_graph(q, k, v, dy, ln, 4, 2, 0.2)
    plain = run(g)[B.NG_MODE_GRAPH_SINGLE]
    if how == "reuse":
        r = GraphRunner(g.workload(), DEV)
        B.ng_set_memory_reuse(r.g, 1)
        try:
            r.prepare(plan_trials=1)
            for mode in (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI):
                r.arena.fill_(0xFF)
                for node, t in g.inputs.items():
                    r.set_input(t, node)
                r.replay(mode)
                for name in plain:
                    assert np.array_equal(r.output(g.names[name]), plain[name]), (mode, name)
        finally:
            r.close()
        return
    got = run(g, MODES, **(dict(launch_fusion=False) if how == "no_fusion" else dict(resident_device_scope=1)))
    for mode, tensors in got.items():
        for name in plain:
            # dk and dv in one launch are cut like each of them alone: the same sums
            assert np.array_equal(tensors[name], plain[name]), (how, mode, name)


def test_replay_after_one_that_gave_up():
    """A device-resident replay whose waits run out of spins leaves arrival counters where they were: the next one starts afresh."""
    q, k, v, dy, ln = attention_inputs(12, 2, 2, 2, 100, 20, 300, None)      # sizes whose kernels are in the resident build
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.25)
    r = GraphRunner(g.workload(), DEV)
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_DEVICE_RESIDENT)
        first = {name: r.output(g.names[name]) for name in ("y", "dq", "dk", "dv")}
        B.ng_resident_config(r.g, 0, 0, 1, 0)                   # one poll: somebody gives up
        r.replay(B.NG_MODE_DEVICE_RESIDENT)
        try:
            r.sync()
        except B.NgError as e:
            assert e.code == B.NG_EHIP
        B.ng_resident_config(r.g, 0, 0, 0, 0)
        for again in (B.ng_replay_static, lambda _: r.replay(B.NG_MODE_DEVICE_RESIDENT), lambda _: r.replay(B.NG_MODE_GRAPH_SINGLE)):
            again(r.g)
            for name in first:
                assert np.array_equal(r.output(g.names[name]), first[name]), name
    finally:
        r.close()
