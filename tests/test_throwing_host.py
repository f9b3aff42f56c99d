"""Nothing throws across the C boundary: with every allocation of a call made to fail in turn, the call returns NG_ENOMEM, and done again it
succeeds with the result of a graph that nothing happened to."""
import json
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NEW = r"""
#include <cstdlib>
#include <new>
static thread_local long left = -1;                             // allocations of this thread until one fails, -1: none does
static void* get(std::size_t n) {
    if (left >= 0 && left-- == 0) throw std::bad_alloc();
    if (void* p = std::malloc(n ? n : 1)) return p;
    throw std::bad_alloc();
}
void* operator new(std::size_t n) { return get(n); }
void* operator new[](std::size_t n) { return get(n); }
void operator delete(void* p) noexcept { std::free(p); }
void operator delete[](void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }
void operator delete[](void* p, std::size_t) noexcept { std::free(p); }
extern "C" void fail_after(long n) { left = n; }
extern "C" long allocations_left() { return left; }
"""

CALLS = r"""
import ctypes, json, sys
new = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)         # ahead of the library: its operator new is the one that is found
import numpy as np
import workloads
from paper_2012_02732_amd import binding as B
from paper_2012_02732_amd.runner import _OPS, _params
new.fail_after.argtypes = [ctypes.c_long]
new.allocations_left.restype = ctypes.c_long
w = workloads.transformer_block(batch=1, layers=1)
out = w.outputs[0]
w = workloads.training_graph(w, 0.1, {out: np.ones(w.nodes[out].shape, np.float32)})
failed = {}

def every(name, call, fails):
    # the call with its first, second, .. allocation failing (every 7th from the 40th on), until none does
    n = 0
    while fails:
        new.fail_after(n)
        try:
            value = call()
            done = True
        except B.NgError as e:
            done = False
            assert e.code == (B.NG_EINVAL if name == "ng_planned_task_kernel" else B.NG_ENOMEM) and "out of host memory" in str(e), str(e)      # (a name is NULL)
        reached = new.allocations_left() < 0
        new.fail_after(-1)
        if done:
            assert not reached, (name, n, "an allocation failed and the call says that nothing did")
            return value
        failed[name] = failed.get(name, 0) + 1
        n += 1 if n < 40 else 7
    return call()

def build(fails):
    g = B.ng_create()
    for nd in w.nodes:
        if nd.op == "input":
            every("ng_add_input", lambda: B.ng_add_input(g, [nd.params[k] for k in "nchw"]), fails)
        else:
            weights = [0] * (len(nd.weights) + len(getattr(nd, "shared_weights", [])))
            every("ng_add_node", lambda: B.ng_add_node(g, _OPS[nd.op], _params(nd), nd.preds, weights), fails)
    for o in w.outputs:
        B.ng_mark_output(g, o)
    every("ng_schedule", lambda: B.ng_schedule(g), fails)
    every("ng_plan_memory", lambda: B.ng_plan_memory(g), fails)
    n = B.ng_num_nodes(g)
    got = [n, [list(B.ng_node_shape(g, v)) for v in range(n)], {k: v for k, v in B.ng_get_schedule(g).items()}]
    got.append(every("ng_get_single_launches", lambda: B.ng_get_single_launches(g), fails))
    got.append(every("ng_get_graph_edges", lambda: B.ng_get_graph_edges(g, 1), fails))
    got.append([every("ng_planned_task_kernel", lambda: B.ng_planned_task_kernel(g, v), fails) for v in (0, n // 2)])
    B.ng_destroy(g)
    return json.loads(json.dumps(got, default=lambda t: t.tolist() if hasattr(t, "tolist") else sorted(t)))

assert build(True) == build(False)
print(json.dumps(failed))
"""


def test_no_memory_is_a_code_and_no_exception(tmp_path):
    (tmp_path / "new.cpp").write_text(NEW)
    lib = str(tmp_path / "new.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", str(tmp_path / "new.cpp"), "-o", lib], check=True)
    (tmp_path / "calls.py").write_text(CALLS)
    done = subprocess.run([sys.executable, str(tmp_path / "calls.py"), lib], cwd=ROOT, capture_output=True, text=True, timeout=300,
                          env=dict(os.environ, PYTHONPATH=ROOT))
    assert done.returncode == 0, (done.returncode, done.stderr[-2000:])
    failed = json.loads(done.stdout.strip().splitlines()[-1])
    assert set(failed) == {"ng_add_input", "ng_add_node", "ng_schedule", "ng_plan_memory", "ng_get_single_launches", "ng_get_graph_edges", "ng_planned_task_kernel"}, failed
