"""Layer norm, dropout and position bias on the GPU against their formulas in 64 bits, in every replay mode. Bounds: block_util.norm_reference
(layer norm, element by element); dropout and the bias are a rounding or two, stated at each test."""
import numpy as np
import pytest
import torch

from attention_util import Graph
from block_util import MODES, U, block_reference, kernels, norm_graph, norm_reference, run, within
from oracle import ops
from oracle.backward import position_bias_vjp
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
F32 = np.float32


def norm_inputs(seed, n, c, h, w, offset=0.5):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, c, h, w)) * (0.5 + 3 * rng.random((1, c, 1, 1))) + offset * rng.standard_normal((1, c, 1, 1))
    return x.astype(F32), rng.uniform(0.5, 1.5, c).astype(F32), rng.standard_normal(c).astype(F32), (rng.standard_normal((n, c, h, w)) * 1e-2).astype(F32)


NORM = [                        # n, c, h, w
    (1, 1, 1, 1), (1, 1, 2, 9), (2, 3, 1, 2), (3, 5, 1, 3), (2, 7, 1, 5), (1, 64, 1, 4), (8, 1024, 1, 1), (5, 1023, 1, 1), (2, 1300, 1, 2), (2, 257, 3, 7), (1, 600, 1, 17), (4, 96, 1, 31),
    (2, 1025, 1, 33), (1, 2048, 2, 8), (1, 4096, 1, 9), (3, 2047, 1, 3), (1, 4097, 1, 3), (2, 5000, 1, 18), (1, 9001, 1, 1), (16, 1100, 1, 259), (130, 4, 1, 37), (700, 40, 1, 6),
    (513, 33, 1, 1), (6, 520, 1, 333), (16, 600, 1, 259), (17, 2100, 1, 255), (40, 700, 1, 300), (3, 3000, 1, 350), (33, 200, 1, 260), (2, 1, 1, 9001),
    (1, 16500, 1, 18), (1, 16384, 1, 21), (3, 12001, 1, 9), (2, 8200, 1, 530), (2, 5121, 1, 2051),
]


@pytest.mark.parametrize("case", NORM, ids=str)
def test_layer_norm(case):
    x, gamma, beta, dy = norm_inputs(1, *case)
    ref = norm_reference(x, gamma, beta, dy, 1e-5)
    g = norm_graph(x, gamma, beta, dy, 1e-5)
    shared = run(g, replays=3)[B.NG_MODE_GRAPH_SINGLE]          # both gradients in one launch
    alone = run(g, launch_fusion=False, replays=2)[B.NG_MODE_GRAPH_SINGLE]
    within(shared, ref, (case, "shared"))
    within(alone, ref, (case, "alone"))
    assert np.array_equal(shared["y"], alone["y"])


@pytest.mark.parametrize("case", [(2, 40, 1, 30), (3, 70, 1, 1), (1, 1500, 1, 40)], ids=str)
def test_layer_norm_in_every_mode(case):
    x, gamma, beta, dy = norm_inputs(2, *case)
    ref = norm_reference(x, gamma, beta, dy, 1e-5)
    forward = run(norm_graph(x, gamma, beta, None, 1e-5), MODES, replays=2)
    assert B.NG_MODE_DEVICE_RESIDENT in forward                 # small tasks have a plan
    for got in (forward, run(norm_graph(x, gamma, beta, dy, 1e-5), MODES, replays=2)):
        assert B.NG_MODE_EAGER_MULTI in got
        for mode, tensors in got.items():
            within(tensors, ref, (case, mode))


def test_layer_norm_of_a_large_mean_and_of_equal_channels():
    x, gamma, beta, dy = norm_inputs(3, 2, 300, 1, 21)
    far = (x + 1000).astype(F32)                                # the variance is 1e-5 of the mean's square
    got = run(norm_graph(far, gamma, beta, dy, 1e-5))[B.NG_MODE_GRAPH_SINGLE]
    within(got, norm_reference(far, gamma, beta, dy, 1e-5), "large mean")
    flat = np.full_like(x, 3.25)                                # sums of 3.25 are exact: nothing is left after the mean
    got = run(norm_graph(flat, gamma, beta, dy, 1e-5))[B.NG_MODE_GRAPH_SINGLE]
    assert np.array_equal(got["y"], np.broadcast_to(beta[None, :, None, None], x.shape))
    within(got, norm_reference(flat, gamma, beta, dy, 1e-5), "equal channels")


def test_layer_norm_of_tensors_beyond_the_caches():
    """The kernels that only large tensors get, against torch in 64 bits on the GPU: 2-norms within the roundings of the formula (mean and
    variance 22 u, three products, a sum over 60001 tokens in parts of 240: sqrt u)."""
    for n, c, t in ((2, 300, 60001), (2, 700, 30003), (1, 3100, 12005), (9, 1000, 3751), (5, 1900, 3606)):
        g = torch.Generator("cuda:0").manual_seed(c)
        x, dy = (torch.randn(n, c, 1, t, generator=g, device="cuda:0") for _ in range(2))
        gamma, beta = (torch.randn(c, generator=g, device="cuda:0") for _ in range(2))
        graph = norm_graph(np.zeros((1, 1, 1, 1), F32), gamma.cpu().numpy(), beta.cpu().numpy(), np.zeros((1, 1, 1, 1), F32), 1e-5)
        for name, value in (("x", x), ("dy", dy)):
            graph.nodes[graph.names[name]].params = dict(n=n, c=c, h=1, w=t)
            graph.inputs[graph.names[name]] = value
        r = GraphRunner(graph.workload(), "cuda:0")
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        leaves = [v.double().requires_grad_() for v in (x, gamma, beta)]
        y = torch.nn.functional.layer_norm(leaves[0].transpose(1, 3), (c,), leaves[1], leaves[2], 1e-5).transpose(1, 3)
        dx, dg, db = torch.autograd.grad(y, leaves, dy.double())
        for name, ref in (("y", y.detach()), ("dx", dx), ("dw", torch.stack([dg, db]).view(2, c, 1, 1))):
            off = float((r.tensor(graph.names[name]).double() - ref).norm() / ref.norm())
            assert off <= 40 * U, (c, name, off / U)
        r.close()


def test_layer_norm_keeps_tokens_apart():
    """A token that is not finite spoils its own results and nothing else of y and dx; the sums over tokens have it."""
    for n, c, h, w in ((2, 40, 1, 10), (2, 40, 1, 3), (1, 4100, 1, 5)):
        x, gamma, beta, dy = norm_inputs(4, n, c, h, w)
        x[0, 7, 0, 2] = np.inf
        x[n - 1, 3, 0, 0] = np.nan
        ref = norm_reference(np.where(np.isfinite(x), x, 0).astype(F32), gamma, beta, dy, 1e-5)
        got = run(norm_graph(x, gamma, beta, dy, 1e-5))[B.NG_MODE_GRAPH_SINGLE]
        good = np.isfinite(x).all(1, keepdims=True) & np.ones_like(x, bool)
        for name in ("y", "dx"):
            off = np.abs(got[name] - ref[name][0])
            assert (off[good] <= ref[name][1][good]).all() and not np.isfinite(got[name][~good]).any(), (n, c, name)


def test_layer_norm_reads_its_weights_on_every_replay_and_writes_its_own_tensor_only():
    x, gamma, beta, dy = norm_inputs(5, 3, 48, 1, 19)
    g = norm_graph(x, gamma, beta, dy, 1e-5)
    r = GraphRunner(g.workload(), "cuda:0")
    r.prepare(plan_trials=1)
    for scale in (1.0, -2.0):
        r.set_weight(g.names["y"], 0, gamma * F32(scale))
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        ref = norm_reference(x, gamma * F32(scale), beta, dy, 1e-5)
        within({name: r.output(g.names[name]) for name in ("y", "dx", "dw")}, ref, scale)
        assert np.array_equal(r.output(g.names["x"]), x) and np.array_equal(r.output(g.names["dy"]), dy)
    r.close()


# ---- dropout -----------------------------------------------------------------------------------------------------------------

def seed_of(*words):
    return np.array(words, np.uint32).view(F32).reshape(1, 1, 1, 2)


def dropout_graph(x, seed, residual, rate, site, dy=None):
    g = Graph()
    g.given("x", x), g.given("seed", seed)
    if residual is not None:
        g.given("residual", residual)
    g.node("y", "dropout", ["x", "seed"] + ([] if residual is None else ["residual"]), np.shape(x), rate=rate, site=site)
    if dy is not None:
        g.given("dy", dy)
        g.node("dx", "dropout", ["dy", "seed"], np.shape(x), rate=rate, site=site)
    return g


def check_dropout(got, x, seed, residual, rate, site, what):
    m = ops.dropout_scale(x.shape, seed, rate, site)
    ref = block_reference("dropout", x, seed, residual, rate, site)
    # the factor, the product and the sum are rounded
    bound = 2 * U * np.abs(x * m) + (0 if residual is None else U * (np.abs(residual) + np.abs(x * m) * (1 + 2 * U)))
    assert (np.abs(got - ref) <= bound).all(), what
    if residual is None:
        assert np.array_equal(got == 0, (m == 0) | (x == 0)), what
    else:
        assert np.array_equal(got[m == 0], residual[m == 0]), what


@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (1, 1, 1, 2), (1, 3, 1, 1), (1, 1, 1, 5), (2, 3, 5, 7), (1, 1, 1, 4095), (1, 4, 32, 32), (1, 1, 1, 4097), (1, 1, 1, 4098), (3, 511, 1, 77), (9, 64, 31, 31)], ids=str)
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(shape, residual):
    rng = np.random.default_rng(sum(shape))
    x, dy, r = (rng.standard_normal(shape).astype(F32) for _ in range(3))
    r = r if residual else None
    for rate, site, seed in ((0.1, 0, seed_of(0, 0)), (0.5, 3, seed_of(0xFFFFFFFF, 0x7FC00001)), (0.0, 2 ** 31 - 1, seed_of(1, 2)), (0.999, 1, seed_of(5, 0x80000000))):
        got = run(dropout_graph(x, seed, r, rate, site, dy), replays=2)[B.NG_MODE_GRAPH_SINGLE]
        check_dropout(got["y"], x, seed, r, rate, site, (shape, rate))
        check_dropout(got["dx"], dy, seed, None, rate, site, (shape, rate, "gradient"))


def test_dropout_in_every_mode_and_new_masks():
    rng = np.random.default_rng(8)
    x, r, dy = (rng.standard_normal((2, 40, 9, 11)).astype(F32) for _ in range(3))
    x[0, 0], r[1, 2] = np.nan, np.inf                           # where they are dropped they are gone; the residual's stay
    seed = seed_of(77, 78)
    got = run(dropout_graph(x, seed, r, 0.5, 4, dy), MODES, replays=2)
    assert B.NG_MODE_DEVICE_RESIDENT in got
    ref = block_reference("dropout", x, seed, r, 0.5, 4)
    for mode, t in got.items():
        assert np.array_equal(np.isfinite(t["y"]), np.isfinite(ref)), mode
        np.testing.assert_allclose(t["y"], ref, rtol=4 * U, atol=4 * U * np.nanmax(np.abs(np.where(np.isfinite(ref), ref, 0))))
        check_dropout(t["dx"], dy, seed, None, 0.5, 4, mode)
    g = dropout_graph(dy, seed, None, 0.5, 4)
    runner = GraphRunner(g.workload(), "cuda:0")
    runner.prepare(plan_trials=1)
    for step in range(3):                                       # the seed is an input like others
        seed = np.array([3.0, step], F32).reshape(1, 1, 1, 2)
        runner.set_input(seed, g.names["seed"])
        runner.replay()
        check_dropout(runner.output(g.names["y"]), dy, seed, None, 0.5, 4, step)
    runner.close()


def test_dropout_in_place_of_a_concat_input():
    """At batch 1 a concat's inputs are written inside its result, at multiples of 16 bytes."""
    rng = np.random.default_rng(9)
    x, seed = rng.standard_normal((1, 4, 3, 3)).astype(F32), seed_of(1, 1)
    g = Graph()
    g.given("x", x), g.given("seed", seed)
    for site in (0, 1):
        g.node(f"y{site}", "dropout", ["x", "seed"], x.shape, rate=0.5, site=site)
    g.node("both", "concat", ["y0", "y1"], (1, 8, 3, 3), lo=[0, 0], hi=[4, 4])
    got = run(g)[B.NG_MODE_GRAPH_SINGLE]
    for site in (0, 1):
        check_dropout(got["both"][:, 4 * site:4 * site + 4], x, seed, None, 0.5, site, site)


def test_dropout_beyond_four_gigabytes():
    n, c, h, w = 5, 64, 2048, 1641                              # 2^30 values and a few
    total = n * c * h * w
    assert total > 2 ** 30
    g = Graph()
    v = g._add("x", __import__("workloads").Node("input", [], dict(n=n, c=c, h=h, w=w), [], (n, c, h, w)))
    g.given("seed", seed_of(9, 10))
    g.inputs[v] = torch.ones(n, c, h, w, device="cuda:0")
    g.node("y", "dropout", ["x", "seed"], (n, c, h, w), rate=0.25, site=6)
    r = GraphRunner(g.workload(), "cuda:0")
    r.prepare(plan_trials=1)
    r.replay(B.NG_MODE_GRAPH_SINGLE)
    r.sync()
    y = r.tensor(g.names["y"]).view(-1)
    limit = 2 ** 30
    for first in (0, 2 ** 29, limit - 4096, limit, total // 4 * 4 - 4096):
        e = np.arange(first // 4, first // 4 + 1024, dtype=np.uint64)
        counter = np.stack([e & np.uint64(0xFFFFFFFF), e >> np.uint64(32), np.full_like(e, 6), np.zeros_like(e)], 1)
        kept = ops.philox4x32(counter, (9, 10)).ravel() >= limit
        got = y[first:first + 4096].cpu().numpy()
        assert np.array_equal(got != 0, kept[:len(got)]) and (np.abs(got[got != 0] - 4 / 3) <= 2 * U * 4 / 3).all(), first
    kept = int((y != 0).sum())
    assert abs(kept - 0.75 * total) <= 6 * np.sqrt(total * 0.75 * 0.25)
    r.close()


# ---- position bias -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,buckets,largest,both", [(1, 4, 2, 1), (3, 8, 10, 1), (16, 32, 128, 1), (5, 32, 128, 0), (2, 2, 2, 0), (7, 64, 1023, 0), (33, 300, 1023, 1)])
def test_position_bias(heads, buckets, largest, both):
    rng = np.random.default_rng(heads)
    table, dbias = rng.standard_normal((buckets, heads)).astype(F32), rng.standard_normal((1, heads, 1, 2 * largest + 1)).astype(F32)
    how = dict(heads=heads, buckets=buckets, max_distance=largest, both=both)
    g = Graph()
    g.given("dbias", dbias)
    g.node("bias", "position_bias", [], dbias.shape, [table], **how)
    g.node("dtable", "position_bias_wgrad", ["dbias"], (buckets, heads, 1, 1), **how)
    got = run(g, MODES, replays=2)
    assert B.NG_MODE_DEVICE_RESIDENT in got
    for mode, t in got.items():
        assert np.array_equal(t["bias"], ops.position_bias(table, heads, buckets, largest, bool(both))), mode
        # a lane adds up every 64th distance of a bucket, then 6 exchanges
        bound = ((2 * largest + 1) / 64 + 8) * U * position_bias_vjp(np.abs(dbias), heads, buckets, largest, bool(both))
        assert (np.abs(t["dtable"][:, :, 0, 0] - position_bias_vjp(dbias, heads, buckets, largest, bool(both))) <= bound).all(), mode
