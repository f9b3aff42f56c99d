"""A graph of the operators around a transformer block's attention has the same bits in every replay mode, whether its gradients share a launch
(one stream) or are launched one by one (several streams, or fusion switched off), and its multi-stream graph passes the check at capture."""
import numpy as np
import pytest

import workloads
from attention_util import attention_graph
from block_util import norm_graph
from test_gpu_biased_attention import LARGE, SMALL, biased_graph, inputs
from test_gpu_block import norm_inputs
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
F32 = np.float32
LAUNCHED = (B.NG_MODE_GRAPH_SINGLE, B.NG_MODE_GRAPH_MULTI, B.NG_MODE_EAGER_SINGLE, B.NG_MODE_EAGER_MULTI)


def same_bits(g, what, together=(), **prepare):
    """`together`: two nodes that share a launch on one stream; returns whether they are on different ones of several. The record of one stream
    is the mode that the others are compared with."""
    got = {}
    apart = False
    for fusion in (True, False):
        r = GraphRunner(g.workload(), "cuda:0")
        try:
            schedule = r.prepare(plan_trials=1, launch_fusion=fusion, **prepare)
            assert B.ng_graph_multi_check(r.g)[0] == 1, (what, fusion, B.ng_graph_multi_check(r.g))
            if together:
                a, b = (g.names[name] for name in together)
                apart = schedule["stream_of"][a] != schedule["stream_of"][b]
            for mode in LAUNCHED:
                r.arena.fill_(0xFF)
                for v, t in g.inputs.items():
                    r.set_input(t, v)
                r.replay(mode)
                r.sync()
                got[fusion, mode] = {name: r.output(v) for name, v in g.names.items() if v not in g.inputs}
        finally:
            r.close()
    first = got[True, B.NG_MODE_GRAPH_SINGLE]
    for mode, tensors in got.items():
        for name, t in tensors.items():
            assert np.isfinite(t).all() and np.array_equal(t.view(np.uint32), first[name].view(np.uint32)), (what, mode, name, int((t != first[name]).sum()), t.size)
    return apart


ONE_BLOCK = [                   # a query's keys are one block of a workgroup that does not split them
    (4, 18, 18, 64, 200, 2, None, 4, "first", "all"),
    (8, 8, 4, 40, 200, 30, "ragged", 12, "last", "all"),
    (1, 6, 6, 96, 540, 4, None, 4, "first", "all"),
]


@pytest.mark.parametrize("case", SMALL[2:5] + SMALL[6:8] + LARGE + ONE_BLOCK, ids=str)
def test_biased_attention(case):
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = case
    args = inputs(9, n, heads, kv, d, tq, tk, lengths, reach, kind)
    same_bits(biased_graph(*args, heads, kv, d ** -0.5, at), case)


def test_dq_and_the_gradient_of_the_bias_on_two_streams():
    """What the cases above are about: one launch on one stream, two launches on two."""
    n, heads, kv, d, tq, tk, lengths, reach, at, kind = LARGE[0]
    g = biased_graph(*inputs(9, n, heads, kv, d, tq, tk, lengths, reach, kind), heads, kv, d ** -0.5, at)
    assert same_bits(g, "apart", together=("dq", "db"))


NORM = [                        # a case of every kernel: 8, half, wide, wide_16, few, many, and a walk of several blocks
    (6, 520, 1, 333), (16, 600, 1, 259), (16, 1100, 1, 259), (17, 2100, 1, 255), (3, 700, 1, 3), (2, 4100, 1, 2), (513, 33, 1, 1), (701, 40, 1, 6), (1, 4096, 1, 9),
]


@pytest.mark.parametrize("case", NORM, ids=str)
def test_layer_norm(case):
    same_bits(norm_graph(*norm_inputs(10, *case), 1e-5), case)


@pytest.mark.parametrize("case", [(2, 6, 2, 64, 257, 333), (2, 4, 4, 128, 300, 520), (3, 4, 4, 64, 33, 64)], ids=str)
def test_attention_without_a_bias(case):
    n, heads, kv, d, tq, tk = case
    q, k, v, dy, _, _ = inputs(11, n, heads, kv, d, tq, tk, None, 1, "all")
    same_bits(attention_graph(q, k, v, dy, None, heads, kv, d ** -0.5), case)


@pytest.mark.parametrize("how", [dict(tokens=70, d=16, layers=1, max_distance=20), dict(tokens=300, d=32, heads=8, kv_heads=4, layers=2, max_distance=40, buckets=12, both=False)], ids=str)
def test_training_of_a_transformer_block(how):
    """A whole step, weights and all, is checked at capture: the multi-stream graph is a mode that the library may pick."""
    w = workloads.transformer_block(batch=2, **how)
    out = w.outputs[0]
    dy = np.random.default_rng(4).standard_normal(w.nodes[out].shape).astype(F32)
    r = GraphRunner(workloads.training_graph(w, 1e-3, {out: dy}), "cuda:0")
    try:
        r.prepare(plan_trials=1)
        assert B.ng_graph_multi_check(r.g)[0] == 1
    finally:
        r.close()
