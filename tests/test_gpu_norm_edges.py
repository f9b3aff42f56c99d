"""Layer norms at the edges of what a kernel holds: as many channels as they have registers for, places without a token where eps is 0. Against
64 bits, element by element (block_util.norm_reference)."""
import pytest

from block_util import norm_graph, norm_reference, run, within
from test_gpu_block import norm_inputs
from paper_2012_02732_amd import binding as B

pytestmark = pytest.mark.gpu


def both_ways(case, eps, seed):
    x, gamma, beta, dy = norm_inputs(seed, *case)
    ref = norm_reference(x, gamma, beta, dy, eps)
    g = norm_graph(x, gamma, beta, dy, eps)
    within(run(g, replays=2)[B.NG_MODE_GRAPH_SINGLE], ref, (case, "shared"))
    within(run(g, launch_fusion=False)[B.NG_MODE_GRAPH_SINGLE], ref, (case, "alone"))


@pytest.mark.parametrize("case", [(2, 1024, 1, 3), (2, 1025, 1, 3), (2, 1100, 1, 3), (1, 1365, 1, 3), (1, 1366, 3, 1), (2, 2048, 1, 2), (2, 2049, 1, 2), (3, 4096, 1, 1), (3, 4097, 1, 1)], ids=str)
def test_few_tokens_of_many_channels(case):
    both_ways(case, 1e-5, 21)


NO_EPS = [                      # places without a token: a fourth lane beside three tokens, and a last round of the walk that some workgroups sit out
    (2, 40, 1, 3), (513, 33, 1, 1), (701, 40, 1, 6), (2, 7, 1, 5), (17, 2100, 1, 271), (19, 1300, 1, 260), (521, 4100, 1, 1), (35, 600, 1, 259),
]


@pytest.mark.parametrize("case", NO_EPS, ids=str)
def test_no_eps(case):
    """With eps = 0 a place without a token has a spread of zero, whose reciprocal must not reach the sums over tokens."""
    both_ways(case, 0.0, 22)
