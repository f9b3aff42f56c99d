"""Attention and its gradients on the GPU within the bounds of their roundings, vector by vector (attention_bounds.py), each case in the
kernels that it names: a case that another choice of kernels would take elsewhere fails here instead of covering nothing."""
import numpy as np
import pytest

from attention_bounds import check
from attention_util import Graph, attention_graph
from test_gpu_attention import attention_inputs, run
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
TILE_64 = {"y": "attention_tile_64", "dq": "attention_dq_tile_64", "dk": "attention_dk_tile_64", "dv": "attention_dv_tile_64"}
TILE_128 = {name: kernel.replace("64", "128") for name, kernel in TILE_64.items()}
WAVE_64 = {name: kernel.replace("tile", "wave") for name, kernel in TILE_64.items()}
WAVE_128 = {name: kernel.replace("64", "128") for name, kernel in WAVE_64.items()}


def kernels(g, unsplit_products=False):
    r = GraphRunner(g.workload())
    try:
        B.ng_set_unsplit_products(r.g, unsplit_products)
        r.schedule()
        r.plan()
        return {name: B.ng_planned_task_kernel(r.g, g.names[name]) for name in ("y", "dq", "dk", "dv") if name in g.names}
    finally:
        r.close()


def forward_graph(q, k, v, heads, kv_heads, scale):
    g = Graph()
    for name, t in (("q", q), ("k", k), ("v", v)):
        g.given(name, t)
    g.node("y", "attention", ["q", "k", "v"], np.shape(q), heads=heads, kv_heads=kv_heads, scale=scale)
    return g


def checked(q, k, v, dy, ln, heads, kv_heads, scale, names, what, unsplit_products=False):
    """Forward and gradients, or without dy the forward operator alone."""
    if dy is None:
        g, names = forward_graph(q, k, v, heads, kv_heads, scale), {"y": names["y"]}
    else:
        g = attention_graph(q, k, v, dy, ln, heads, kv_heads, scale)
    assert kernels(g, unsplit_products) == names, (what, kernels(g, unsplit_products))
    got = run(g, unsplit_products=unsplit_products)[B.NG_MODE_GRAPH_SINGLE]
    check(got, q, k, v, dy, ln, heads, kv_heads, scale, what)
    return got


@pytest.mark.parametrize("case,names", [
    ((3, 8, 4, 128, 150, 333, "ragged"), TILE_128),
    ((2, 6, 2, 100, 171, 777, "odd"), TILE_128),
    ((1, 4, 1, 128, 33, 6000, None), TILE_128),                 # few queries, many keys: split over the keys
    ((1, 2, 2, 128, 2100, 200, None), TILE_128),                # many queries, few keys: dk and dv split over the queries
    ((2, 4, 2, 64, 300, 500, "ragged"), TILE_64),
    ((1, 8, 1, 40, 50, 2000, "odd"), TILE_64),
    ((6, 8, 8, 33, 257, 129, "ragged"), TILE_64),
    ((2, 4, 2, 64, 33, 31, "ragged"), WAVE_64),
    ((5, 4, 2, 128, 19, 63, "odd"), WAVE_128),
    ((1, 2, 1, 65, 2, 4099, None), WAVE_128),
], ids=str)
def test_attention_and_gradients_vector_by_vector(case, names):
    n, heads, kv_heads, d, tq, tk, kind = case
    q, k, v, dy, ln = attention_inputs(tq + 7 * tk, n, heads, kv_heads, d, tq, tk, kind)
    checked(q, k, v, dy, ln, heads, kv_heads, d ** -0.5, names, case)


def grown(t, powers):
    """Token by token times 2^0 .. 2^powers."""
    return (t * 2.0 ** np.round(np.linspace(0, powers, t.shape[3]))).astype(np.float32)


@pytest.mark.parametrize("which", ["keys", "queries", "values", "values_shrink", "dy", "keys_at_once", "values_at_once", "sharp", "negative"])
@pytest.mark.parametrize("sizes,names", [((2, 8, 4, 128, 150, 333), TILE_128), ((2, 8, 4, 64, 150, 333), TILE_64)], ids=["128", "64"])
def test_attention_of_magnitudes_that_change_along_the_tokens(sizes, names, which):
    """What is summed so far is brought to a new reference score or unit, often or by much at once."""
    n, heads, kv_heads, d, tq, tk = sizes
    q, k, v, dy, ln = attention_inputs(21, n, heads, kv_heads, d, tq, tk, None)
    scale = d ** -0.5
    late = np.ones(tk, np.float32)
    if which == "keys":
        k = grown(k, 3)
    elif which == "queries":
        q = grown(q, 3)
    elif which == "values":
        v = grown(v, 20)
    elif which == "values_shrink":
        v = grown(v, -12)
    elif which == "dy":
        dy = grown(dy, 12)
    elif which == "keys_at_once":
        late[200:] = 8.0
        k = k * late
    elif which == "values_at_once":
        late[200:] = 2.0 ** 30
        v = v * late
    else:
        scale = 4.0 if which == "sharp" else -scale
    checked(q, k, v, dy, ln, heads, kv_heads, scale, names, (sizes, which))


@pytest.mark.parametrize("sizes,names", [((1, 2, 2, 64, 512, 100), dict(TILE_64, y="attention_wave_64", dq="attention_dq_wave_64")),
                                         ((1, 8, 8, 64, 512, 200), TILE_64), ((1, 8, 4, 128, 512, 200), TILE_128)], ids=str)
def test_dv_of_keys_that_get_little_weight(sizes, names):
    """Every query gives some keys 2^-20 .. 2^-40 of its largest weight: their dv is as precise, of its own size, as the others'."""
    n, heads, kv_heads, d, tq, tk = sizes
    q, k, v, dy, ln = attention_inputs(31, n, heads, kv_heads, d, tq, tk, None)
    q[:, ::d] = 4.0                                             # channel 0 of every head
    k[:, ::d] = 0.0
    k[:, ::d, :, -40:] = -2.0 * np.log(2.0) * np.repeat([20, 28, 32, 40], 10)       # 4 k / 8 = -ln 2 of that
    checked(q, k, v, dy, ln, heads, kv_heads, 0.125, names, sizes)


def test_dv_of_queries_with_sharp_and_with_even_weights():
    """Some queries give all their weight to one key, the others the same to each of 16384; dy of the former is 2^12 times as large.
    The keys that only the latter read have a dv as precise as ever."""
    d, tq, tk = 64, 128, 16384
    q, k, v, dy, ln = attention_inputs(41, 1, 1, 1, d, tq, tk, None)
    q *= np.float32(0.1)
    q[:, 1], k[:, 1] = 0.0, 0.0
    q[:, 1, :, ::2], k[:, 1, :, 0] = 8.0, 64.0
    dy[:, :, :, ::2] *= 2.0 ** 12
    checked(q, k, v, dy, ln, 1, 1, 0.125, TILE_64, "sharp and even")


def test_attention_of_zero_queries_with_a_tiny_scale():
    """Queries of zeros weigh all keys alike whatever the scale is; the last block has keys that do not exist."""
    for d, names in ((64, TILE_64), (128, TILE_128)):
        q, k, v, dy, ln = attention_inputs(51, 2, 8, 4, d, 150, 333, None)
        q[:, :, :, ::3] = 0.0
        k[:, : d] = 0.0
        checked(q, k, v, dy, ln, 8, 4, 1e-9, names, d)


@pytest.mark.parametrize("q_size,k_size,scale_size", [(2.0 ** -60, 2.0 ** -50, 2.0 ** 110), (2.0 ** -70, 2.0 ** -50, 2.0 ** 120), (2.0 ** 60, 2.0 ** 50, 2.0 ** -110)])
def test_attention_of_products_that_the_scale_makes_up_for(q_size, k_size, scale_size):
    for d, names in ((64, TILE_64), (128, TILE_128)):
        q, k, v, dy, ln = attention_inputs(61, 2, 8, 4, d, 150, 333, None)
        q, k = q * np.float32(q_size), k * np.float32(k_size)
        checked(q, k, v, dy, ln, 8, 4, d ** -0.5 * scale_size, names, (d, q_size))


@pytest.mark.parametrize("case,names", [((1, 4, 4, 64, 40, 5000), TILE_64), ((1, 4, 1, 128, 33, 6000), TILE_128), ((2, 8, 4, 128, 150, 333), TILE_128)], ids=str)
def test_attention_of_values_next_to_the_largest(case, names):
    """Weighted means of values of 2^120: no sum on the way leaves fp32's range, cut into splits or not."""
    n, heads, kv_heads, d, tq, tk = case
    q, k, v, dy, ln = attention_inputs(71, n, heads, kv_heads, d, tq, tk, None)
    v = (np.abs(v) * 2.0 ** 120).astype(np.float32)
    checked(q, k, v, None, ln, heads, kv_heads, d ** -0.5, names, case)


@pytest.mark.parametrize("sizes,names", [((2, 8, 4, 128, 150, 333), WAVE_128), ((2, 8, 4, 64, 150, 333), WAVE_64), ((1, 4, 4, 64, 40, 5000), WAVE_64)], ids=str)
@pytest.mark.parametrize("powers", [-30, 30])
def test_unsplit_products_of_channels_of_very_different_size(sizes, names, powers):
    """Channels 2^0 .. 2^powers as large as the first, made up for in the factor that they meet: with products of fp32 values, of this size
    too, every vector is as precise as ever (in half-precision parts the small ones lose their bits)."""
    n, heads, kv_heads, d, tq, tk = sizes
    q, k, v, dy, ln = attention_inputs(81, n, heads, kv_heads, d, tq, tk, None)
    each = (2.0 ** np.round(np.linspace(0, powers, d))).astype(np.float32)
    per_q, per_k = (np.tile(each, m)[None, :, None, None] for m in (heads, kv_heads))
    checked(q, k, v * per_k, dy / per_q, ln, heads, kv_heads, d ** -0.5, names, (sizes, powers, "values"), unsplit_products=True)
    checked(q * per_q, k / per_k, v, dy, ln, heads, kv_heads, d ** -0.5, names, (sizes, powers, "keys"), unsplit_products=True)


def test_unsplit_products_are_chosen_before_binding():
    q, k, v, dy, ln = attention_inputs(81, 1, 2, 2, 16, 4, 5, None)
    r = GraphRunner(attention_graph(q, k, v, dy, ln, 2, 2, 0.25).workload(), "cuda:0")
    try:
        r.prepare(plan_trials=1)
        with pytest.raises(B.NgError) as e:
            B.ng_set_unsplit_products(r.g, True)
        assert e.value.code == B.NG_ESTATE
    finally:
        r.close()
