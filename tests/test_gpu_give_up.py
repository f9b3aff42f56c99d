"""The first replay after a device-resident one that gave up, in every mode: arrival counts that it left are not counted on."""
import numpy as np
import pytest

from attention_util import attention_graph
from test_gpu_attention import DEV, attention_inputs
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
MODES = {"graph_multi": B.NG_MODE_GRAPH_MULTI, "graph_single": B.NG_MODE_GRAPH_SINGLE, "eager_single": B.NG_MODE_EAGER_SINGLE,
         "eager_multi": B.NG_MODE_EAGER_MULTI, "resident": B.NG_MODE_DEVICE_RESIDENT, "static": None}


def replay(r, mode):
    if MODES[mode] is None:
        B.ng_replay_static(r.g)
    else:
        r.replay(MODES[mode])


def give_up(r, static=False):
    """A replay with one poll: whoever waits for anything gives up."""
    B.ng_resident_config(r.g, 0, 0, 1, 0)
    if static:
        B.ng_replay_static(r.g)
    else:
        r.replay(B.NG_MODE_DEVICE_RESIDENT)
    B.ng_resident_config(r.g, 0, 0, 0, 0)


@pytest.mark.parametrize("static", [False, True], ids=["replay", "static"])
@pytest.mark.parametrize("asked", [True, False], ids=["reported", "not_asked"])
@pytest.mark.parametrize("mode", list(MODES))
def test_first_replay_after_one_that_gave_up(mode, asked, static):
    """``asked``: ng_sync has reported it before the next replay. Otherwise the error is still there to be reported, and the replay is
    right all the same."""
    import torch
    q, k, v, dy, ln = attention_inputs(12, 2, 2, 2, 100, 20, 300, None)      # sizes whose kernels are in the resident build, split
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.25)
    r = GraphRunner(g.workload(), DEV)
    names = ("y", "dq", "dk", "dv")
    try:
        r.prepare(plan_trials=1)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        first = {name: r.output(g.names[name]) for name in names}
        for turn in range(3):
            give_up(r, static)
            if asked:
                with pytest.raises(B.NgError) as e:
                    r.sync()
                assert e.value.code == B.NG_EHIP
            else:
                torch.cuda.synchronize(DEV)
            for name in names:
                r.tensor(g.names[name]).fill_(float("nan"))
            torch.cuda.synchronize(DEV)
            for again in range(2):                              # the counts are whole after it as well
                replay(r, mode)
                if asked or again:
                    r.sync()                                    # nothing of the one that gave up is reported for this one
                else:
                    with pytest.raises(B.NgError) as e:         # the report that nobody had asked for
                        r.sync()
                    assert e.value.code == B.NG_EHIP
                for name in names:
                    got = r.tensor(g.names[name]).cpu().numpy()
                    assert np.array_equal(got, first[name]), (turn, again, name)
    finally:
        r.close()


def test_report_stays_until_the_next_replay():
    q, k, v, dy, ln = attention_inputs(12, 2, 2, 2, 100, 20, 300, None)
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.25)
    r = GraphRunner(g.workload(), DEV)
    try:
        r.prepare(plan_trials=1)
        give_up(r)
        for _ in range(2):
            with pytest.raises(B.NgError) as e:
                r.sync()
            assert e.value.code == B.NG_EHIP and "ran out of spins" in str(e.value)
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
        r.sync()
    finally:
        r.close()


def test_check_of_the_multi_stream_graph_after_one_that_gave_up():
    """ng_graph_multi_recheck compares two modes: counts left over must not make them differ."""
    q, k, v, dy, ln = attention_inputs(12, 2, 2, 2, 100, 20, 300, None)
    g = attention_graph(q, k, v, dy, ln, 2, 2, 0.25)
    r = GraphRunner(g.workload(), DEV)
    try:
        r.prepare(plan_trials=1)
        assert B.ng_graph_multi_check(r.g)[0] == 1
        give_up(r)
        with pytest.raises(B.NgError):
            r.sync()
        B.ng_graph_multi_recheck(r.g, 4)
        assert B.ng_graph_multi_check(r.g)[0] == 1
        r.replay(B.NG_MODE_GRAPH_SINGLE)
        r.sync()
    finally:
        r.close()


def test_a_refused_replay_does_not_end_the_report():
    q, k, v, dy, ln = attention_inputs(12, 2, 2, 2, 100, 20, 300, None)
    r = GraphRunner(attention_graph(q, k, v, dy, ln, 2, 2, 0.25).workload(), DEV)
    try:
        r.prepare(plan_trials=1)
        B.ng_graph_multi_distrust(r.g)
        give_up(r)
        for _ in range(2):
            with pytest.raises(B.NgError) as e:
                r.sync()
            assert e.value.code == B.NG_EHIP
            with pytest.raises(B.NgError) as e:
                r.replay(B.NG_MODE_GRAPH_MULTI)
            assert e.value.code == B.NG_ESTATE
        r.replay(B.NG_MODE_EAGER_SINGLE)
        r.sync()
    finally:
        r.close()


@pytest.mark.parametrize("mode", list(MODES))
def test_gradients_of_convolutions_after_one_that_gave_up(mode):
    """The sums by last arrival of convolutions, depthwise convolutions and batch-norms; a rate of 0 leaves the weights as they are."""
    import workloads
    w = workloads.nas_cell_cifar(batch=4, image=16)
    out = w.outputs[0]
    seed = np.random.default_rng(1).standard_normal(w.nodes[out].shape).astype(np.float32)
    tw = workloads.training_graph(w, 0.0, {out: seed})
    r = GraphRunner(tw, DEV)
    try:
        r.prepare(plan_trials=1)
        grads = sorted({node for node, _, _ in tw.wgrad_of.values()})
        replay(r, mode)
        first = {node: r.output(node) for node in grads}
        for _ in range(2):
            give_up(r)
            with pytest.raises(B.NgError) as e:
                r.sync()
            assert e.value.code == B.NG_EHIP
            for _ in range(2):
                replay(r, mode)
                for node in grads:
                    assert np.array_equal(r.output(node), first[node]), (mode, node, tw.nodes[node].op)
    finally:
        r.close()
