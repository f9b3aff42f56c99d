"""Layer norm of images of millions of pixels, every element against 64 bits: a workgroup's registers hold more channels than these images have,
and the places of those that do not exist lie beyond 2^31 bytes."""
import numpy as np
import pytest
import torch

from block_util import U
from test_gpu_attention_calls import on_device
from paper_2012_02732_amd import GraphRunner, binding as B

pytestmark = pytest.mark.gpu
DEV, F32 = "cuda:0", np.float32


@pytest.mark.parametrize("c,h,w", [(8, 4096, 4096), (64, 2048, 2048), (2, 1, 3000001), (128, 1, 2500000), (520, 1, 1000000), (1100, 1, 480001)], ids=str)
def test_layer_norm_of_a_long_image(c, h, w):
    """y and dx element by element with the bounds of block_util.norm_reference. The sums over T tokens by 2-norm: a thread adds up n = T / 256 + 4
    of them at most (four at a time, at least 256 workgroups of at least 4 tokens), each addition off by u of what there is by then, which
    for terms of both signs is sqrt(n / 2) u of the sum; the sums of these sums, 8 u; a token's xh is off by e_xh, independently of the others'."""
    t, eps = h * w, float(F32(1e-5))
    assert c * t <= 1 << 29
    g = torch.Generator(DEV).manual_seed(c)
    x, dy = (torch.randn(1, c, h, w, generator=g, device=DEV) for _ in range(2))
    gamma, beta = np.linspace(0.5, 1.5, c).astype(F32), np.linspace(-1, 1, c).astype(F32)
    ops = [("y", "layer_norm", ["x"], x.shape, dict(eps=1e-5), [gamma, beta], []),
           ("dx", "layer_norm_dgrad", ["dy", "x"], x.shape, dict(eps=1e-5), [], [("y", 0), ("y", 1)]),
           ("dw", "layer_norm_wgrad", ["dy", "x"], (2, c, 1, 1), dict(eps=1e-5), [], [("y", 0), ("y", 1)])]
    gm, bt = (torch.from_numpy(v).to(DEV).double()[:, None] for v in (gamma, beta))
    S = max(16, c / 16) + 22
    for fusion in (True, False):                                # both gradients in one launch, and one by one
        workload, ids = on_device(dict(x=x, dy=dy), ops)
        r = GraphRunner(workload, DEV)
        try:
            r.prepare(plan_trials=1, launch_fusion=fusion)
            for name in ("y", "dx", "dw"):
                r.tensor(ids[name]).fill_(float("nan"))
            torch.cuda.synchronize(DEV)                         # (the replay is on a stream of its own)
            r.replay(B.NG_MODE_GRAPH_SINGLE)
            r.sync()
            sums, squares = torch.zeros(2, c, dtype=torch.float64, device=DEV), 0.0
            step = (1 << 24) // c
            for first in range(0, t, step):
                xs, gs = (v.view(c, t)[:, first:first + step].double() for v in (x, dy))
                s = (xs.var(0, unbiased=False) + eps).sqrt()
                xh, a = (xs - xs.mean(0)) / s, xs.abs().mean(0)
                e_xh = U * (S * a / s * (1 + xh.abs()) + (S / 2 + 7) * xh.abs())
                u = gs * gm
                m1, m2 = u.mean(0), (u * xh).mean(0)
                off1 = (S + 2) * U * u.abs().mean(0)
                off2 = (S + 3) * U * (u * xh).abs().mean(0) + (u.abs() * e_xh).mean(0)
                inside = 3 * U * u.abs() + off1 + 3 * U * m1.abs() + xh.abs() * off2 + m2.abs() * e_xh + 4 * U * (xh * m2).abs()
                may = {"y": gm * e_xh + 4 * U * ((gm * xh).abs() + bt.abs()),
                       "dx": (inside + U * (S * a / s + S / 2 + 8) * (u.abs() + m1.abs() + (xh * m2).abs())) / s}
                for name, ref in (("y", gm * xh + bt), ("dx", (u - m1 - xh * m2) / s)):
                    off = (r.tensor(ids[name]).view(c, t)[:, first:first + step].double() - ref).abs()
                    assert bool((off <= may[name]).all()), (fusion, name, first, int((~(off <= may[name])).sum()))
                sums += torch.stack([(gs * xh).sum(1), gs.sum(1)])
                squares += float(((gs * e_xh) ** 2).sum())
            off = float((r.tensor(ids["dw"]).view(2, c).double() - sums).norm())
            may = (8 + (t / 512 + 2) ** 0.5) * U * float(sums.norm()) + squares ** 0.5
            assert off <= may, (fusion, off / may)
        finally:
            r.close()
