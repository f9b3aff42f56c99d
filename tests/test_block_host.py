"""Layer norm, dropout and position bias without a GPU: shapes, refusals, the work that is reported, the kernels that are chosen."""
import numpy as np
import pytest

import workloads
from block_util import kernels, norm_graph
from paper_2012_02732_amd import GraphRunner, binding as B


class G:
    def __init__(self, **inputs):
        self.g = B.ng_create()
        self.id = {name: B.ng_add_input(self.g, shape) for name, shape in inputs.items()}

    def add(self, op, preds, n_weights=0, **values):
        p = B.ng_op_params()
        for name, v in values.items():
            setattr(p, name, v)
        return B.ng_add_node(self.g, op, p, [self.id.get(u, u) for u in preds], [0] * n_weights)

    def shape(self, *args, **values):
        return tuple(B.ng_node_shape(self.g, self.add(*args, **values)))

    def refused(self, code, text, *args, **values):
        before = B.ng_num_nodes(self.g)
        with pytest.raises(B.NgError) as e:
            self.add(*args, **values)
        assert e.value.code == code and text in str(e.value), str(e.value)
        assert B.ng_num_nodes(self.g) == before


def test_layer_norm_shapes_and_refusals():
    g = G(x=(2, 12, 3, 5), turned=(2, 12, 5, 3), huge=(1, 1 << 20, 1, 1024))
    fwd, dgrad, wgrad = B.NG_OP_LAYER_NORM, B.NG_OP_LAYER_NORM_DGRAD, B.NG_OP_LAYER_NORM_WGRAD
    assert g.shape(fwd, ["x"], 2, eps=1e-5) == (2, 12, 3, 5) and g.shape(fwd, ["x"], 2, eps=0.0) == (2, 12, 3, 5)
    assert g.shape(dgrad, ["x", "x"], 2, eps=1e-5) == (2, 12, 3, 5) and g.shape(wgrad, ["x", "x"], 2, eps=1e-5) == (2, 12, 1, 1)
    for op, preds in ((fwd, ["x"]), (dgrad, ["x", "x"]), (wgrad, ["x", "x"])):
        for eps in (-1.0, float("nan"), float("inf")):
            g.refused(B.NG_EINVAL, "eps", op, preds, 2, eps=eps)
        for n_weights in (0, 1, 3):
            g.refused(B.NG_EINVAL, "gamma and beta", op, preds, n_weights)
    g.refused(B.NG_EINVAL, "layer_norm takes", fwd, ["x", "x"], 2)
    g.refused(B.NG_EINVAL, "layer_norm backward takes", dgrad, ["x"], 2)
    g.refused(B.NG_ESHAPE, "differ", dgrad, ["turned", "x"], 2)
    g.refused(B.NG_ESHAPE, "differ", wgrad, ["turned", "x"], 2)
    g.refused(B.NG_ESHAPE, "2^29", fwd, ["huge"], 2)
    B.ng_destroy(g.g)


def test_dropout_shapes_and_refusals():
    g = G(x=(2, 12, 3, 5), seed=(1, 1, 1, 2), tall=(1, 1, 2, 1), other=(2, 12, 5, 3))
    drop = B.NG_OP_DROPOUT
    for rate in (0.0, 0.5, 1 - 2.0 ** -24):
        assert g.shape(drop, ["x", "seed"], rate=rate) == g.shape(drop, ["x", "seed", "x"], rate=rate, site=2 ** 31 - 1) == (2, 12, 3, 5)
    assert g.shape(drop, ["seed", "seed"], rate=0.5) == (1, 1, 1, 2)
    for rate in (1.0, -0.1, float("nan"), float("inf")):
        g.refused(B.NG_EINVAL, "rate", drop, ["x", "seed"], rate=rate)
    g.refused(B.NG_EINVAL, "site", drop, ["x", "seed"], site=-1)
    g.refused(B.NG_EINVAL, "dropout takes", drop, ["x"])
    g.refused(B.NG_EINVAL, "dropout takes", drop, ["x", "seed", "x", "x"])
    g.refused(B.NG_EINVAL, "dropout takes", drop, ["x", "seed"], 1)
    g.refused(B.NG_ESHAPE, "seed", drop, ["x", "tall"])
    g.refused(B.NG_ESHAPE, "seed", drop, ["x", "x"])
    g.refused(B.NG_ESHAPE, "residual", drop, ["x", "seed", "other"])
    B.ng_destroy(g.g)


def test_position_bias_shapes_and_refusals():
    g = G(x=(1, 4, 1, 21), other=(1, 4, 21, 1))
    op, wgrad = B.NG_OP_POSITION_BIAS, B.NG_OP_POSITION_BIAS_WGRAD
    how = dict(heads=4, buckets=8, max_distance=10, both=1)
    assert g.shape(op, [], 1, **how) == (1, 4, 1, 21)
    assert g.shape(wgrad, ["x"], **how) == (8, 4, 1, 1)
    assert g.shape(op, [], 1, heads=1, buckets=2, max_distance=2, both=0) == (1, 1, 1, 5)
    for bad in (dict(heads=0), dict(both=2), dict(buckets=2), dict(buckets=7), dict(buckets=0), dict(max_distance=1024), dict(max_distance=2), dict(max_distance=-1),
                dict(both=0, buckets=1), dict(both=0, max_distance=4), dict(heads=2 ** 21), dict(buckets=2 ** 21)):
        g.refused(B.NG_EINVAL, "position_bias", op, [], 1, **dict(how, **bad))
        g.refused(B.NG_EINVAL, "position_bias", wgrad, ["x"], **dict(how, **bad))
    g.refused(B.NG_EINVAL, "position_bias takes", op, ["x"], 1, **how)
    g.refused(B.NG_EINVAL, "position_bias takes", op, [], **how)
    g.refused(B.NG_ESHAPE, "position_bias_wgrad", wgrad, ["other"], **how)
    g.refused(B.NG_ESHAPE, "position_bias_wgrad", wgrad, ["x"], **dict(how, heads=2))
    g.refused(B.NG_EINVAL, "predecessors", wgrad, [], **how)      # only the bias itself has none
    g.refused(B.NG_EINVAL, "predecessors", B.NG_OP_RELU, [])
    B.ng_destroy(g.g)


def test_a_graph_that_begins_with_a_bias_is_planned():
    """A task that waits for nothing: scheduled, placed and given launches like the others."""
    g = G(x=(1, 4, 1, 21))
    b = g.add(B.NG_OP_POSITION_BIAS, [], 1, heads=4, buckets=8, max_distance=10, both=1)
    s = g.add(B.NG_OP_ADD_N, ["x", b])
    B.ng_mark_output(g.g, s)
    B.ng_schedule(g.g)
    B.ng_plan_memory(g.g)
    assert B.ng_planned_task_kernel(g.g, b) == "position_bias"
    assert B.ng_resident_dry_plan(g.g)["ok"]
    assert (b, s) in B.ng_get_graph_edges(g.g, 0)[1]
    B.ng_destroy(g.g)


def test_work_of_the_block_operators():
    g = G(x=(2, 12, 3, 5), seed=(1, 1, 1, 2))
    n = 2 * 12 * 15
    for op, preds, weights, how, expected in ((B.NG_OP_LAYER_NORM, ["x"], 2, {}, 4 * (2 * n + 24)), (B.NG_OP_LAYER_NORM_DGRAD, ["x", "x"], 2, {}, 4 * (3 * n + 24)),
                                              (B.NG_OP_LAYER_NORM_WGRAD, ["x", "x"], 2, {}, 4 * (2 * n + 24)), (B.NG_OP_DROPOUT, ["x", "seed"], 0, {}, 4 * (2 * n + 2)),
                                              (B.NG_OP_DROPOUT, ["x", "seed", "x"], 0, {}, 4 * (3 * n + 2)),
                                              (B.NG_OP_POSITION_BIAS, [], 1, dict(heads=2, buckets=4, max_distance=5, both=1), 4 * (22 + 8))):
        assert B.ng_task_work(g.g, g.add(op, preds, weights, **how))[0] == expected, op
    B.ng_destroy(g.g)


NORM_KERNELS = [                # n, c, h, w, name of the forward kernel, what the gradients' end in
    (8, 1024, 1, 1, "layer_norm_few", "few"), (2, 7, 1, 3, "layer_norm_few", "few"), (1, 2000, 1, 3, "layer_norm_many", "many"), (1, 4097, 1, 1, "layer_norm_many", "many"),
    (2, 5000, 1, 18, "layer_norm_half_16", "wide"), (1, 16385, 1, 18, "layer_norm_many", "many"), (1, 16384, 1, 21, "layer_norm_wide_16", "wide_16"), (1, 4097, 1, 9, "layer_norm_half_16", "wide"), (6, 520, 1, 333, "layer_norm_8", "8"), (2, 33, 3, 7, "layer_norm_8", "8"), (1, 2048, 2, 8, "layer_norm_8", "8"),
    (1, 4096, 1, 4, "layer_norm_16", "half"), (16, 600, 1, 259, "layer_norm_half", "half"), (16, 1100, 1, 300, "layer_norm_half_16", "wide"), (16, 2100, 1, 259, "layer_norm_wide_16", "wide_16"),
    (2, 4096, 1, 8192, "layer_norm_wide_16", "wide_16"), (8, 1024, 1, 4096, "layer_norm_half", "wide"), (16, 1024, 1, 4096, "layer_norm_half_16", "wide"), (16, 512, 1, 8192, "layer_norm_half", "half"),
]


@pytest.mark.parametrize("case", NORM_KERNELS, ids=str)
def test_kernels_of_layer_norm(case):
    n, c, h, w, name, gradients = case
    x = np.broadcast_to(np.float32(0), (n, c, h, w))
    g = norm_graph(np.zeros((1, 1, 1, 1), np.float32), np.zeros(1, np.float32), np.zeros(1, np.float32), np.zeros((1, 1, 1, 1), np.float32), 1e-5)
    for nd in g.nodes[:1] + [g.nodes[g.names["dy"]]]:           # the shapes alone
        nd.params = dict(zip("nchw", x.shape))
    found = kernels(g)
    assert found["y"] == name
    assert found["dx"] == f"layer_norm_dgrad_{gradients}" and found["dw"] == f"layer_norm_wgrad_{gradients}"


def test_gradients_of_a_norm_share_a_launch():
    g = norm_graph(*(np.zeros(s, np.float32) for s in ((2, 40, 1, 30), 40, 40, (2, 40, 1, 30))), 1e-5)
    for fused, launches in ((True, 2), (False, 3)):
        r = GraphRunner(g.workload())
        if not fused:
            B.ng_set_launch_fusion(r.g, False)
        r.schedule(), r.plan()
        assert B.ng_get_single_launches(r.g)[1] == launches
        r.close()


def test_training_graph_of_a_transformer_block():
    for both in (True, False):
        w = workloads.transformer_block(both=both)
        out = w.outputs[0]
        tw = workloads.training_graph(w, 0.01, {out: np.ones(w.nodes[out].shape, np.float32)})
        ops = [nd.op for nd in tw.nodes]
        assert ops.count("layer_norm_dgrad") == 3 and ops.count("layer_norm_wgrad") == 4       # nothing below the first norm has a gradient
        assert ops.count("dropout") == 8 and ops.count("attention_dbias") == 2 and ops.count("position_bias_wgrad") == 1
        assert {(v, j) for v, nd in enumerate(w.nodes) for j in range(len(nd.weights))} == set(tw.update_of)


def test_biased_attention_shapes_and_refusals():
    g = G(q=(2, 32, 1, 5), k=(2, 16, 3, 3), ln=(2, 1, 1, 1), bias=(1, 4, 1, 7), even=(1, 4, 1, 6), heads2=(1, 2, 1, 7), tall=(1, 4, 7, 1), each=(2, 4, 1, 7),
          wide=(1, 4, 1, 2049), dy=(2, 32, 1, 5), one=(1, 4, 1, 1))
    att, rows_op, db = B.NG_OP_ATTENTION, B.NG_OP_ATTENTION_ROWS, B.NG_OP_ATTENTION_DBIAS
    how = dict(heads=4, kv_heads=2, scale=0.5, bias=1)
    y = g.add(att, ["q", "k", "k", "bias"], **how)
    z = g.add(att, ["q", "k", "k", "ln", "bias"], **dict(how, bias=2))
    plain = g.add(att, ["q", "k", "k", "ln"], **dict(how, bias=0))
    assert g.shape(att, ["q", "k", "k", "one"], **how) == (2, 32, 1, 5)
    rows, rows2, rows0 = (g.add(rows_op, ["dy", v], **how) for v in (y, z, plain))
    for op, shape in ((B.NG_OP_ATTENTION_DQ, (2, 32, 1, 5)), (B.NG_OP_ATTENTION_DK, (2, 16, 3, 3)), (B.NG_OP_ATTENTION_DV, (2, 16, 3, 3)), (db, (1, 4, 1, 7))):
        assert g.shape(op, ["dy", rows, "q", "k", "k", "bias"], **how) == shape
        assert g.shape(op, ["dy", rows2, "q", "k", "k", "ln", "bias"], **dict(how, bias=2)) == shape
        g.refused(B.NG_EINVAL, "rows are of an attention", op, ["dy", rows2, "q", "k", "k", "ln", "bias"], **how)        # aligned otherwise
        g.refused(B.NG_EINVAL, "rows are of an attention", op, ["dy", rows0, "q", "k", "k", "bias"], **how)
        g.refused(B.NG_EINVAL, "attention", op, ["dy", rows, "q", "k", "k"], **how)
        g.refused(B.NG_EINVAL, "bias in", op, ["dy", rows, "q", "k", "k", "bias"], **dict(how, bias=3))
    g.refused(B.NG_EINVAL, "no bias", db, ["dy", rows0, "q", "k", "k", "ln"], **dict(how, bias=0))
    for bad in ("even", "heads2", "tall", "each", "wide", "ln"):
        g.refused(B.NG_ESHAPE, "the bias must be", att, ["q", "k", "k", bad], **how)
    g.refused(B.NG_ESHAPE, "lengths", att, ["q", "k", "k", "bias"], **dict(how, bias=0))
    g.refused(B.NG_ESHAPE, "lengths", att, ["q", "k", "k", "bias", "bias"], **how)
    for value in (-1, 3):
        g.refused(B.NG_EINVAL, "bias in", att, ["q", "k", "k", "bias"], **dict(how, bias=value))
    g.refused(B.NG_EINVAL, "attention takes", att, ["q", "k", "k"], **how)
    assert B.ng_task_work(g.g, y)[0] == 4 * (320 + 2 * 288 + 320 + 28)
    B.ng_destroy(g.g)
