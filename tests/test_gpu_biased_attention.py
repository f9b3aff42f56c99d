"""Attention with a bias of distances on the GPU against its formulas in 64 bits: kernels for few and for many columns, lengths, shared heads,
masks, and all gradients.

Tolerances, u = 2^-24. A score is a sum of d products, times the scale, plus the bias, in units of log2: with S the largest sum of magnitudes
scale |q| |k| and B the largest bias it is off by e = u ((d + 10) S + 6 B), and every softmax weight by 2 e of itself.
  y, dq, dk, dv  as in test_gpu_attention.py, with these weights
  dbias          terms p (dp - <dy, y>) are off by (2 e + (2 d + 16) u) of p (|dy| |v| + sum p |dy| |v|); they are added up 32 to a diagonal, then
                 over the blocks of keys, then over rows in groups of 16: (Tk / 32 + 120) u of the sum of these magnitudes
"""
import numpy as np
import pytest

import workloads
from attention_util import Graph
from block_util import U, kernels, run
from oracle import ops
from oracle.backward import attention_vjp
from oracle.forward import forward
from paper_2012_02732_amd import GraphRunner, binding as B
from test_gpu_attention import lengths_of, norm_off

pytestmark = pytest.mark.gpu
F32 = np.float32
MODES = (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_SINGLE, B.NG_MODE_EAGER_MULTI)


def biased_graph(q, k, v, dy, ln, bias, heads, kv_heads, scale, at, which=("dq", "dk", "dv", "db")):
    g = Graph()
    for name, t in (("q", q), ("k", k), ("v", v), ("bias", bias)):
        g.given(name, t)
    last = []
    if ln is not None:
        g.given("lengths", ln)
        last = ["lengths"]
    last += ["bias"]
    how = dict(heads=heads, kv_heads=kv_heads, scale=scale, bias=at)
    g.node("y", "attention", ["q", "k", "v"] + last, np.shape(q), **how)
    if dy is not None:
        g.given("dy", dy)
        g.node("rows", "attention_rows", ["dy", "y"], heads=heads)
        for name in which:
            g.node(name, "attention_dbias" if name == "db" else "attention_" + name, ["dy", "rows", "q", "k", "v"] + last, **how)
    return g


def bias_of(kind, rng, heads, reach):
    b = rng.standard_normal((1, heads, 1, 2 * reach + 1)).astype(F32) * 2
    far = np.arange(-reach, reach + 1)
    if kind == "back":                                          # only looks back
        b[..., far > 0] = -np.inf
    elif kind == "window":                                      # near keys only; one head sees everything
        b[..., np.abs(far) >= max(reach, 1)] = -np.inf
        if heads > 1:
            b[0, 1] = rng.standard_normal(2 * reach + 1)
    elif kind == "ahead":                                       # only later keys: the last queries see none
        b[..., far <= 0] = -np.inf
    elif kind == "holes":
        b[rng.random(b.shape) < 0.5] = -np.inf
    elif kind == "nothing":
        b[...] = -np.inf
    else:
        assert kind == "all"
    return b


def inputs(seed, n, heads, kv_heads, d, tq, tk, lengths, reach, kind):
    rng = np.random.default_rng(seed)
    q, dy = (rng.standard_normal((n, heads * d, 1, tq)).astype(F32) for _ in range(2))
    k, v = (rng.standard_normal((n, kv_heads * d, 1, tk)).astype(F32) for _ in range(2))
    ln = lengths_of(lengths, n, tk)
    if ln is not None:
        for b in range(n):
            m = ops.key_count(float(ln[b, 0, 0, 0]), tk)
            k[b, :, :, m:], v[b, :, :, m:] = np.nan, np.inf
    return q, k, v, dy, ln, bias_of(kind, rng, heads, reach)


def check(got, q, k, v, dy, ln, bias, heads, kv_heads, scale, at, what):
    n, d, tq, tk = q.shape[0], q.shape[1] // heads, q.shape[3], k.shape[3]
    scale = float(F32(scale))
    k, v = (np.where(np.isfinite(t), t, 0).astype(np.float64) for t in (k, v))
    group = heads // kv_heads
    p = ops.attention_weights(q, k, heads, kv_heads, scale, ln, bias, at)
    vh = ops.counted_values(v, kv_heads, ln)
    y = np.stack([np.stack([vh[b, h // group] @ p[b, h].T for h in range(heads)]) for b in range(n)]).reshape(q.shape)
    qa, ka = np.abs(q.reshape(n, kv_heads, group, d, tq)).astype(np.float64), np.abs(k.reshape(n, kv_heads, 1, d, tk))
    S = abs(scale) * (qa.transpose(0, 1, 2, 4, 3) @ ka).max()
    top = np.abs(bias[np.isfinite(bias)]).max(initial=0.0)
    e = U * ((d + 10) * S + 6 * top)
    assert np.isfinite(got["y"]).all(), what
    off = np.abs(got["y"] - y).max()
    assert off <= (2 * e + (tk + 8) * U) * np.abs(v).max(), (what, "y", off)
    spread = max(1.0, abs(scale) * d ** 0.5)
    assert not y.any() or norm_off(got["y"], y) <= 4 * (np.sqrt(d) * spread + np.sqrt(min(tk, 256)) + 8 + 2 * top) * U, (what, "y", norm_off(got["y"], y))
    seen = p.sum(3).transpose(0, 1, 2).reshape(n, heads, 1, tq) > 0
    assert not got["y"].reshape(n, heads, d, tq)[~np.broadcast_to(seen, (n, heads, d, tq))].any(), (what, "a query without a key")
    if "rows" not in got:
        return
    grads = dict(zip(("dq", "dk", "dv", "db"), attention_vjp(q, k, v, ln, heads, kv_heads, scale, dy, bias, at)))
    largest = max(d, tk, group * tq)
    tol = 4 * (2 * np.sqrt(d) * spread + 2 * np.sqrt(min(largest, 1024)) + 16 + 4 * top) * U
    gy = np.linalg.norm(dy.astype(np.float64).reshape(n, heads, d, tq), axis=2)
    for name, other in (("dq", k), ("dk", q.astype(np.float64))):
        if name in got:
            size = abs(scale) * np.sqrt(d) * np.abs(v).max() * np.abs(other).max() * np.sqrt((gy ** 2).sum())
            off = np.linalg.norm(got[name] - grads[name])
            assert np.isfinite(got[name]).all() and off <= tol * max(size, 1e-300), (what, name, off, tol * size)
            # (queries that see one key have dS = 0 whatever the inputs: nothing to be relative to where there are only these)
            assert np.linalg.norm(grads[name]) <= 1e-3 * size or norm_off(got[name], grads[name]) <= 100 * tol, (what, name, norm_off(got[name], grads[name]))
    if "dv" in got:
        size = np.linalg.norm(attention_vjp(q, k, v, ln, heads, kv_heads, scale, np.abs(dy), bias, at)[2])
        assert np.isfinite(got["dv"]).all() and np.linalg.norm(got["dv"] - grads["dv"]) <= tol * max(size, 1e-300), (what, "dv")
    if "db" in got:
        mag = np.zeros_like(grads["db"])[0, :, 0]
        reach = mag.shape[1] // 2
        ya, va = np.abs(dy.astype(np.float64)).reshape(n, heads, d, tq), np.abs(vh)
        for b in range(n):
            m = tk if ln is None else ops.key_count(float(ln[b, 0, 0, 0]), tk)
            for h in range(heads):
                t = ya[b, h].T @ va[b, h // group]
                t = p[b, h] * (t + (p[b, h] * t).sum(1, keepdims=True))
                np.add.at(mag[h], ops.distances(tq, m, reach, m - tq if at == "last" else 0), t[:, :m])
        bound = (2 * e + (2 * d + 16) * U + (tk / 32 + 120) * U) * mag
        off = np.abs(got["db"][0, :, 0] - grads["db"][0, :, 0])
        assert (off <= bound).all(), (what, "db", float(off.max()), float((off / np.maximum(bound, 1e-300)).max()))
    if ln is not None:
        for b in range(n):
            m = ops.key_count(float(ln[b, 0, 0, 0]), tk)
            assert all(not got[name][b, :, :, m:].any() for name in ("dk", "dv") if name in got), (what, b)


SMALL = [                       # n, heads, kv_heads, d, Tq, Tk, lengths, reach, at, kind
    (1, 1, 1, 1, 1, 1, None, 0, "first", "all"),
    (2, 2, 1, 8, 1, 3, "odd", 1, "last", "all"),
    (5, 2, 2, 16, 3, 5, "odd", 2, "last", "back"),
    (2, 4, 2, 40, 17, 77, None, 5, "first", "all"),
    (5, 8, 1, 64, 1, 200, "ragged", 128, "last", "back"),
    (1, 3, 3, 7, 5, 129, None, 1023, "first", "all"),
    (3, 4, 4, 64, 33, 64, "ragged", 16, "first", "back"),
    (1, 2, 2, 128, 130, 65, None, 40, "last", "window"),
    (5, 4, 2, 128, 19, 63, "odd", 64, "first", "holes"),
    (2, 16, 2, 100, 1, 1030, "ragged", 1000, "last", "window"),
    (2, 4, 4, 33, 70, 20, None, 3, "last", "back"),
    (2, 3, 3, 64, 40, 50, "ragged", 30, "first", "ahead"),
    (1, 2, 1, 16, 20, 30, None, 4, "first", "nothing"),
    (1, 2, 1, 65, 2, 4099, None, 128, "last", "window"),
    (3, 6, 3, 24, 4, 300, "ragged", 0, "last", "all"),
]
LARGE = [
    (2, 6, 2, 64, 257, 333, "ragged", 128, "first", "all"),
    (2, 6, 2, 64, 257, 333, "ragged", 128, "last", "back"),
    (2, 4, 4, 128, 300, 520, None, 128, "first", "all"),
    (2, 4, 4, 128, 300, 520, None, 50, "last", "back"),
    (3, 8, 4, 40, 129, 700, "ragged", 7, "first", "back"),
    (2, 8, 8, 64, 500, 500, None, 33, "first", "window"),
    (2, 8, 8, 96, 500, 400, None, 1023, "last", "holes"),
    (4, 8, 2, 64, 150, 640, "odd", 20, "last", "ahead"),
    (1, 8, 8, 64, 600, 600, None, 300, "first", "nothing"),
    (1, 4, 4, 64, 1111, 1030, None, 0, "first", "all"),
    (1, 2, 1, 128, 1025, 1500, None, 128, "last", "back"),
    (2, 8, 8, 64, 700, 300, None, 64, "last", "back"),          # the first queries come before every key
]


@pytest.mark.parametrize("case", SMALL + LARGE, ids=str)
def test_biased_attention_and_its_gradients(case):
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = case
    args = inputs(1, n, heads, kv, d, tq, tk, lengths, reach, kind)
    scale = d ** -0.5
    got = run(biased_graph(*args, heads, kv, scale, at), replays=3)[B.NG_MODE_GRAPH_SINGLE]
    check(got, *args, heads, kv, scale, at, (case, "shared launches"))
    alone = run(biased_graph(*args, heads, kv, scale, at), launch_fusion=False)[B.NG_MODE_GRAPH_SINGLE]
    check(alone, *args, heads, kv, scale, at, (case, "alone"))


@pytest.mark.parametrize("case", LARGE[:6], ids=str)
def test_biased_attention_without_parts(case):
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = case
    args = inputs(2, n, heads, kv, d, tq, tk, lengths, reach, kind)
    got = run(biased_graph(*args, heads, kv, d ** -0.5, at), unsplit_products=True)[B.NG_MODE_GRAPH_SINGLE]
    check(got, *args, heads, kv, d ** -0.5, at, case)


@pytest.mark.parametrize("case", [SMALL[2], SMALL[6], LARGE[1], LARGE[3]], ids=str)
@pytest.mark.parametrize("scale", [-0.3, 1.5])
def test_biased_attention_in_every_mode(case, scale):
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = case
    args = inputs(3, n, heads, kv, d, tq, tk, lengths, reach, kind)
    got = run(biased_graph(*args, heads, kv, scale * d ** -0.5, at), MODES, replays=2)
    assert B.NG_MODE_EAGER_MULTI in got
    for mode, t in got.items():
        check(t, *args, heads, kv, scale * d ** -0.5, at, (case, mode))


@pytest.mark.parametrize("which", [("db",), ("dq",), ("dk",), ("dv",), ("dv", "db"), ("db", "dq", "dk")], ids=str)
def test_gradients_by_themselves(which):
    for case in (LARGE[0], LARGE[3], SMALL[8]):
        n, heads, kv, d, tq, tk, lengths, reach, at, kind = case
        args = inputs(4, n, heads, kv, d, tq, tk, lengths, reach, kind)
        check(run(biased_graph(*args, heads, kv, d ** -0.5, at, which))[B.NG_MODE_GRAPH_SINGLE], *args, heads, kv, d ** -0.5, at, (case, which))


def test_kernels_of_the_cases():
    """The cases above run the kernels they are meant for."""
    names = set()
    for n, heads, kv, d, tq, tk, lengths, reach, at, kind in SMALL + LARGE:
        names |= set(kernels(biased_graph(*inputs(1, n, heads, kv, d, tq, tk, lengths, reach, kind), heads, kv, 1.0, at)).values())
    for base in ("attention_biased", "attention_biased_dq", "attention_biased_dk", "attention_biased_dv", "attention_dbias"):
        for how in ("wave_64", "wave_128", "tile_64", "tile_128"):
            assert f"{base}_{how}" in names, (base, how, sorted(names))


@pytest.mark.parametrize("case", [(2, 2, 2, 64, 40, 70, 8), (2, 8, 8, 64, 300, 333, 8), (2, 8, 4, 128, 300, 333, 8)], ids=str)
def test_masks_of_the_lowest_value(case):
    """The lowest finite value hides a key from queries that have others; queries with nothing else have the mean of these keys, whose
    scores the value has taken up (3.4e38 plus a score of ten is 3.4e38)."""
    n, heads, kv, d, tq, tk, reach = case
    q, k, v, dy, ln, bias = inputs(5, n, heads, kv, d, tq, tk, "ragged", reach, "all")
    bias[..., np.arange(-reach, reach + 1) <= 0] = np.finfo(F32).min       # the last queries have no key ahead
    got = run(biased_graph(q, k, v, dy, ln, bias, heads, kv, d ** -0.5, "first"))[B.NG_MODE_GRAPH_SINGLE]
    assert all(np.isfinite(t).all() for t in got.values())
    # the reference's scores plus the bias in 64 bits are the bias to 2^-53 of it: the same mean
    clean = bias.copy()
    p = ops.attention_weights(q, np.where(np.isfinite(k), k, 0), heads, kv, d ** -0.5, ln, clean, "first")
    vh = ops.counted_values(np.where(np.isfinite(v), v, 0), kv, ln)
    y = np.stack([np.stack([vh[b, h // (heads // kv)] @ p[b, h].T for h in range(heads)]) for b in range(n)]).reshape(q.shape)
    S = 4 * d ** 0.5                                            # scores of normal values stay below that
    assert np.abs(got["y"] - y).max() <= (2 * U * ((d + 10) * S + 6 * 8) + (tk + 8) * U) * np.abs(vh).max()
    grads = dict(zip(("dq", "dk", "dv", "db"), attention_vjp(q, np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0), ln, heads, kv, d ** -0.5, dy, clean, "first")))
    for name, t in grads.items():
        assert norm_off(got[name], t) <= 400 * (2 * np.sqrt(d) + 2 * np.sqrt(1024) + 16 + 40) * U, (name, norm_off(got[name], t))


def test_biases_beyond_what_a_shared_number_may_be():
    """Blocks beyond the reach, all of one bias of 1e5: the scores are rounded to its bits (2^-7), in the gradients as in the weights."""
    n, heads, kv, d, tq, tk, reach = 1, 4, 4, 64, 512, 640, 2
    q, k, v, dy, ln, bias = inputs(6, n, heads, kv, d, tq, tk, None, reach, "all")
    near = run(biased_graph(q, k, v, dy, ln, bias, heads, kv, d ** -0.5, "first"))[B.NG_MODE_GRAPH_SINGLE]
    got = run(biased_graph(q, k, v, dy, ln, (bias + F32(1e5)).astype(F32), heads, kv, d ** -0.5, "first"))[B.NG_MODE_GRAPH_SINGLE]
    # softmax does not see a number added to all scores; each is off by half a step at 1.5e5 in units of log2, 2^-8, the bias by 2^-8 of a unit before
    for name in ("y", "dq", "dk", "dv"):
        assert norm_off(got[name], near[name]) <= 8 * 2.0 ** -7, (name, norm_off(got[name], near[name]))


def test_a_bias_of_zeros_changes_nothing():
    from attention_util import attention_graph
    n, heads, kv, d, tq, tk = 2, 4, 2, 64, 300, 333
    q, k, v, dy, ln, bias = inputs(7, n, heads, kv, d, tq, tk, "ragged", 64, "all")
    got = run(biased_graph(q, k, v, dy, ln, np.zeros_like(bias), heads, kv, d ** -0.5, "last"))[B.NG_MODE_GRAPH_SINGLE]
    plain = run(attention_graph(q, k, v, dy, ln, heads, kv, d ** -0.5))[B.NG_MODE_GRAPH_SINGLE]
    for name in ("y", "dq", "dk", "dv"):
        assert norm_off(got[name], plain[name]) <= 4 * (4 * np.sqrt(d) + 2 * 32 + 24) * U, name


def test_one_tensor_in_every_place_and_a_bias_read_twice():
    """q = k = v, and two attentions that read one bias: its gradients are summed by the graph."""
    n, heads, d, t, reach = 2, 4, 32, 90, 20
    q, _, _, dy, _, bias = inputs(8, n, heads, heads, d, t, t, None, reach, "back")
    g = Graph()
    for name, x in (("x", q), ("bias", bias), ("dy", dy)):
        g.given(name, x)
    how = dict(heads=heads, kv_heads=heads, scale=0.2, bias="first")
    for i in "12":
        g.node("y" + i, "attention", ["x", "x", "x", "bias"], q.shape, **how)
        g.node("rows" + i, "attention_rows", ["dy", "y" + i], heads=heads)
        g.node("db" + i, "attention_dbias", ["dy", "rows" + i, "x", "x", "x", "bias"], **how)
        g.node("dq" + i, "attention_dq", ["dy", "rows" + i, "x", "x", "x", "bias"], **how)
    g.node("db", "add_n", ["db1", "db2"], bias.shape)
    got = run(g, MODES, replays=2)
    for mode, t in got.items():
        check({"y": t["y1"], "rows": t["rows1"], "db": t["db1"], "dq": t["dq1"]}, q, q, q, dy, None, bias, heads, heads, 0.2, "first", mode)
        assert np.array_equal(t["db1"], t["db2"]) and np.array_equal(t["db"], 2 * t["db1"])


def test_no_device_resident_plan():
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = SMALL[3]
    g = biased_graph(*inputs(1, n, heads, kv, d, tq, tk, lengths, reach, kind), heads, kv, 1.0, at)
    r = GraphRunner(g.workload(), "cuda:0")
    r.prepare(plan_trials=1)
    for call in (lambda: r.replay(B.NG_MODE_DEVICE_RESIDENT), lambda: B.ng_replay_static(r.g)):
        with pytest.raises(B.NgError) as e:
            call()
        assert e.value.code == B.NG_ESTATE and "no device-resident plan" in str(e.value)
    r.close()


# ---- together ----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("how", [dict(), dict(both=False), dict(tokens=150, d=32, layers=1, max_distance=40, buckets=12, lengths=[150, 0])], ids=str)
def test_a_transformer_block_is_trained(how):
    """Forward, all gradients and the update of a block of these operators, against the oracle's; then steps with other masks."""
    from oracle.backward import backward, sgd_step
    w = workloads.transformer_block(batch=2, **how)
    out = w.outputs[0]
    rng = np.random.default_rng(4)
    dy = rng.standard_normal(w.nodes[out].shape).astype(F32)
    lr = 1e-3
    tw = workloads.training_graph(w, lr, {out: dy})
    r = GraphRunner(tw, "cuda:0")
    r.prepare(plan_trials=1)
    key = w.nodes[[v for v, nd in enumerate(w.nodes) if nd.op == "dropout"][0]].preds[1]
    for step in range(2):
        seed = np.array([11, step], F32).reshape(1, 1, 1, 2)
        w.inputs[key] = seed
        r.set_input(seed, key)
        for v, nd in enumerate(w.nodes):                        # the weights as they are before this step
            nd.weights = [r.weight(v, j) for j in range(len(nd.weights))]
        val = forward(w)[out]
        d_value, d_weight = backward(w, {out: dy})
        r.replay()
        assert np.abs(r.output(out) - val).max() <= 1e-4 * np.abs(val).max()
        for v, nd in enumerate(w.nodes):
            for j, keep in enumerate(nd.weights):
                new = r.weight(v, j)
                ref = sgd_step([keep], [np.reshape(d_weight[v][j], keep.shape)], lr)[0]
                moved = np.abs(ref.astype(np.float64) - keep).max()
                assert np.abs(new - ref).max() <= 1e-3 * moved + 4 * U * np.abs(keep).max(), (step, v, nd.op, j)
    r.close()
