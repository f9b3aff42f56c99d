"""Attention operators without a GPU: shapes, refusals, the work that is reported, the kernels that are chosen, the training graph."""
import numpy as np
import pytest

import workloads
from oracle.backward import backward
from oracle.forward import forward
from paper_2012_02732_amd import GraphRunner, binding as B


def params(**values):
    p = B.ng_op_params()
    for name, v in dict(dict(heads=2, kv_heads=2, rot=4, scale=0.5, factor=1.0, eps=1e-6), **values).items():
        setattr(p, name, v)
    return p


class G:
    def __init__(self, **inputs):
        self.g = B.ng_create()
        self.id = {name: B.ng_add_input(self.g, shape) for name, shape in inputs.items()}

    def add(self, op, preds, n_weights=0, **values):
        return B.ng_add_node(self.g, op, params(**values), [self.id.get(p, p) for p in preds], [0] * n_weights)

    def refused(self, code, text, op, preds, n_weights=0, **values):
        before = B.ng_num_nodes(self.g)
        with pytest.raises(B.NgError) as e:
            self.add(op, preds, n_weights, **values)
        assert e.value.code == code and text in str(e.value), str(e.value)
        assert B.ng_num_nodes(self.g) == before


def test_head_rope_shapes_and_refusals():
    g = G(x=(2, 12, 3, 5), pos=(1, 1, 3, 5), each=(2, 1, 3, 5), row=(1, 1, 1, 15), wide=(1, 514, 1, 4), pos4=(1, 1, 1, 4), dy=(2, 12, 5, 3))
    rope, dgrad, wgrad = B.NG_OP_HEAD_ROPE, B.NG_OP_HEAD_ROPE_DGRAD, B.NG_OP_HEAD_ROPE_WGRAD
    y = g.add(rope, ["x", "pos"], 2)
    assert tuple(B.ng_node_shape(g.g, y)) == (2, 12, 3, 5)
    assert tuple(B.ng_node_shape(g.g, g.add(rope, ["x", "each"], 1, rot=6, interleaved=1))) == (2, 12, 3, 5)
    assert tuple(B.ng_node_shape(g.g, g.add(dgrad, [y, "x", "pos"], 1))) == (2, 12, 3, 5)
    assert tuple(B.ng_node_shape(g.g, g.add(wgrad, [y, "x", "pos"], 2))) == (1, 6, 1, 1)
    for bad in (dict(heads=0), dict(heads=5), dict(heads=-2), dict(rot=0), dict(rot=3), dict(rot=8), dict(rot=-2), dict(interleaved=2),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(factor=float("nan")), dict(factor=float("inf")), dict(factor=0.0)):
        g.refused(B.NG_EINVAL, "head_rope", rope, ["x", "pos"], 2, **bad)
    g.refused(B.NG_EINVAL, "256", rope, ["wide", "pos4"], 1, heads=2)
    for n_weights in (0, 3):
        g.refused(B.NG_EINVAL, "weights", rope, ["x", "pos"], n_weights)
    g.refused(B.NG_EINVAL, "head_rope backward", wgrad, [y, "x", "pos"], 1)
    g.refused(B.NG_EINVAL, "head_rope backward", dgrad, [y, "x"], 1)
    g.refused(B.NG_ESHAPE, "positions", rope, ["x", "row"], 2)
    g.refused(B.NG_ESHAPE, "positions", rope, ["x", "x"], 2)
    g.refused(B.NG_ESHAPE, "differ", dgrad, ["dy", "x", "pos"], 1)
    B.ng_destroy(g.g)


def test_attention_shapes_and_refusals():
    g = G(q=(2, 32, 1, 5), k=(2, 16, 3, 3), v=(2, 16, 3, 3), ln=(2, 1, 1, 1), ln1=(1, 1, 1, 1), other=(2, 16, 1, 9), one=(1, 16, 3, 3), dy=(2, 32, 1, 5),
          big=(1, 258, 1, 4))
    how = dict(heads=4, kv_heads=2)
    att, rows_op = B.NG_OP_ATTENTION, B.NG_OP_ATTENTION_ROWS
    y = g.add(att, ["q", "k", "v"], **how)
    yl = g.add(att, ["q", "k", "v", "ln"], **how)
    assert tuple(B.ng_node_shape(g.g, yl)) == (2, 32, 1, 5)
    rows = g.add(rows_op, ["dy", y], **how)
    assert tuple(B.ng_node_shape(g.g, rows)) == (2, 12, 1, 5)
    for op, shape in ((B.NG_OP_ATTENTION_DQ, (2, 32, 1, 5)), (B.NG_OP_ATTENTION_DK, (2, 16, 3, 3)), (B.NG_OP_ATTENTION_DV, (2, 16, 3, 3))):
        assert tuple(B.ng_node_shape(g.g, g.add(op, ["dy", rows, "q", "k", "v"], **how))) == shape
        g.refused(B.NG_EINVAL, "rows are of an attention", op, ["dy", rows, "q", "k", "v", "ln"], **how)      # of the one without lengths
        g.refused(B.NG_EINVAL, "rows are of an attention", op, ["dy", rows, "q", "v", "k"], **how)
        g.refused(B.NG_EINVAL, "rows are of an attention", op, ["dy", rows, "q", "k", "v"], scale=0.25, **how)
        g.refused(B.NG_EINVAL, "attention_rows node of dy", op, ["q", rows, "q", "k", "v"], **how)
        g.refused(B.NG_EINVAL, "attention_rows node of dy", op, ["dy", y, "q", "k", "v"], **how)
        g.refused(B.NG_EINVAL, "takes dy, rows", op, ["dy", rows, "q", "k"], **how)
    for bad in (dict(heads=4, kv_heads=3), dict(heads=0, kv_heads=1), dict(heads=4, kv_heads=0), dict(heads=4, kv_heads=-2), dict(heads=4, kv_heads=2, scale=float("inf")),
                dict(heads=4, kv_heads=2, scale=float("nan")), dict(heads=4, kv_heads=2, scale=0.0),
                dict(heads=4, kv_heads=2, scale=3e38)):        # finite, but not times log2 e
        g.refused(B.NG_EINVAL, "attention", att, ["q", "k", "v"], **bad)
    g.refused(B.NG_ESHAPE, "128", att, ["big", "big", "big"], heads=2, kv_heads=2)
    g.refused(B.NG_ESHAPE, "heads must divide", att, ["q", "k", "v"], heads=5, kv_heads=5)
    g.refused(B.NG_ESHAPE, "k and v", att, ["q", "k", "other"], **how)
    g.refused(B.NG_ESHAPE, "k and v", att, ["q", "one", "one"], **how)
    g.refused(B.NG_ESHAPE, "k and v", att, ["q", "k", "v"], heads=4, kv_heads=4)
    g.refused(B.NG_ESHAPE, "lengths", att, ["q", "k", "v", "ln1"], **how)
    g.refused(B.NG_EINVAL, "takes q, k, v", att, ["q", "k"], **how)
    g.refused(B.NG_EINVAL, "takes q, k, v", att, ["q", "k", "v"], 1, **how)
    g.refused(B.NG_EINVAL, "must be an attention node", rows_op, ["dy", "q"], **how)
    g.refused(B.NG_EINVAL, "must be an attention node", rows_op, ["dy", y], heads=2)
    g.refused(B.NG_ESHAPE, "differ", rows_op, ["k", y], **how)
    B.ng_destroy(g.g)


def test_extents_beyond_32_bit_offsets_and_launches_are_refused():
    long = 1 << 24
    most = 1 << 22
    g = G(q=(1, 256, 1, 4), k=(1, 128, 1, most), ks=(1, 32, 1, most), qs=(1, 32, 1, 4), kl=(1, 32, 1, most + 1), long=(1, 2048, 1, 1 << 19), k4=(1, 64, 1, 4), x=(1, 64, 1, long), pos=(1, 1, 1, long), tiny=(1 << 23, 1, 1, 1))
    assert g.add(B.NG_OP_ATTENTION, ["q", "k", "k"], heads=2, kv_heads=1) > 0
    g.refused(B.NG_ESHAPE, "2^22", B.NG_OP_ATTENTION, ["qs", "kl", "kl"], heads=1, kv_heads=1)
    g.refused(B.NG_ESHAPE, "2^29", B.NG_OP_ATTENTION, ["long", "k4", "k4"], heads=32, kv_heads=1)      # the heads of q that read one of k
    assert g.add(B.NG_OP_ATTENTION, ["qs", "ks", "ks"], heads=1, kv_heads=1) > 0
    g.refused(B.NG_ESHAPE, "2^29", B.NG_OP_HEAD_ROPE, ["x", "pos"], 1, heads=1, rot=2)
    g.refused(B.NG_ESHAPE, "too many", B.NG_OP_ATTENTION, ["tiny", "tiny", "tiny"], heads=1, kv_heads=1)
    B.ng_destroy(g.g)


def test_training_graph_of_a_block_with_attention():
    w = workloads.decoder_block()
    out = w.outputs[0]
    seed = np.random.default_rng(1).standard_normal(w.nodes[out].shape).astype(np.float32)
    tw = workloads.training_graph(w, 0.01, {out: seed})
    assert {v for v in tw.inputs} == {0, 1, 2, 3, 4, len(w.nodes)}
    ops = [nd.op for nd in tw.nodes]
    assert ops.count("attention_rows") == 2 and ops.count("attention_dq") == ops.count("attention_dk") == ops.count("attention_dv") == 2
    assert ops.count("head_rope_dgrad") == 3 and ops.count("head_rope_wgrad") == 2
    assert {(v, j) for v, nd in enumerate(w.nodes) for j in range(len(nd.weights)) if not (nd.op == "head_rope" and j == 0)} == set(tw.update_of)
    for mode in ("host",):
        r = GraphRunner(tw)                                     # the library infers the shapes that the recipe expects
        for v, nd in enumerate(tw.nodes):
            assert tuple(B.ng_node_shape(r.g, v)) == tuple(nd.shape), (v, nd.op)
            B.ng_task_work(r.g, v)
        r.schedule()
        r.plan()
        names = {nd.op: B.ng_planned_task_kernel(r.g, v) for v, nd in enumerate(tw.nodes)}
        assert names["attention"] and names["head_rope_wgrad"].startswith("head_rope_wgrad"), names
        r.close()
    d_value, d_weight = backward(w, {out: seed})                # finite differences of the whole block, in its weights
    val = forward(w)[out]
    assert np.isfinite(val).all() and np.isfinite(d_value[0]).all()
    conv = next(v for v, nd in enumerate(w.nodes) if nd.op == "conv1x1" and nd.preds == [1])
    at, step, side = (1, 2), 1e-2, []
    for sgn in (1, -1):
        keep = w.nodes[conv].weights[0].copy()
        w.nodes[conv].weights[0][at] += sgn * step
        side.append(float((forward(w)[out].astype(np.float64) * seed).sum()))
        w.nodes[conv].weights[0] = keep
    # a second-order difference of a smooth function: step^2 of the third derivative, and fp32 storage between the operators
    assert abs((side[0] - side[1]) / (2 * step) - d_weight[conv][0][at]) <= 1e-2 * max(1.0, np.abs(d_weight[conv][0]).max())


def test_work_of_attention():
    g = G(q=(2, 32, 1, 5), k=(2, 16, 1, 9), pos=(1, 1, 1, 5))
    y = g.add(B.NG_OP_ATTENTION, ["q", "k", "k"], heads=4, kv_heads=2)
    nbytes, flops = B.ng_task_work(g.g, y)
    assert nbytes == 4 * (320 + 2 * 288 + 320) and flops == 2 * 2 * 320 * 9
    r = g.add(B.NG_OP_HEAD_ROPE, ["q", "pos"], 2, heads=4)
    assert B.ng_task_work(g.g, r)[0] == 4 * (2 * 320 + 5)
    B.ng_destroy(g.g)


def test_device_resident_plan_of_attention():
    """Small tasks have a plan; a graph with kernels that the attention build does not have is refused rather than planned."""
    few = G(q=(1, 64, 1, 8), k=(1, 64, 1, 300), pos=(1, 1, 1, 8))
    y = few.add(B.NG_OP_HEAD_ROPE, ["q", "pos"], 1, heads=2)
    few.add(B.NG_OP_ATTENTION, [y, "k", "k"], heads=2, kv_heads=2)
    many = G(q=(1, 64, 1, 2048), k=(1, 64, 1, 2048))
    many.add(B.NG_OP_ATTENTION, ["q", "k", "k"], heads=2, kv_heads=2)
    for g, planned in ((few, True), (many, False)):
        B.ng_mark_output(g.g, B.ng_num_nodes(g.g) - 1)
        B.ng_schedule(g.g)
        B.ng_plan_memory(g.g)
        if planned:
            assert B.ng_resident_dry_plan(g.g)["ok"]
        else:
            with pytest.raises(B.NgError) as e:
                B.ng_resident_dry_plan(g.g)
            assert e.value.code == B.NG_ESTATE and "no device-resident plan" in str(e.value)
        B.ng_destroy(g.g)
