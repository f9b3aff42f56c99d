"""Attention operators of the DAG executor as timed cases: what a network with attention asks of them, and what they compute.

Tensors are fp32 and channel-major, as the 1 x 1 convolutions around these operators leave and take them: [n][heads * d][1][T],
the T tokens of an image (a sequence) contiguous. Four operators, each a node of a graph:

head_rope            x [n][H d][1][T], positions [1 or n][1][1][T], frequencies f[rot / 2], gamma[d] (without it: no norm)
                       u = x * gamma / sqrt(mean over the head's d channels of x^2 + eps)
                       (a, b) = factor * (a cos - b sin, a sin + b cos) at the angle position * f[i], for the pairs i of the head's
                       first rot channels: (2 i, 2 i + 1) interleaved, (i, i + rot / 2) otherwise; the other channels are u
head_rope backward   dx and dgamma from dy
attention            q [n][H d][1][Tq], k, v [n][Hk d][1][Tk], lengths [n]; query head h reads key head h / (H / Hk)
                       p[i][j] = softmax over j < lengths[image] of scale * <q_i, k_j>; y_i = sum_j p[i][j] v_j; without a key: 0
attention backward   dq, dk, dv from dy

A pass of a training case is the forward operator and its gradients, as one graph. The framework's side keeps a captured graph whose
inputs lie in its arena, as every program of this framework does, and replays it.
"""
import dataclasses
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6


def listed():
    return [
        # ---- norm of queries or keys for each head, and their rotation ----
        # one new token for each of 8 sequences, far into them: the smallest call, all of it latency
        _rope("rope_token", n=8, heads=16, d=64, rot=64, T=1, start=30000, spread=1),
        # prompts of a batch, a quarter of each head rotated, interleaved pairs, no norm
        _rope("rope_partial", n=4, heads=16, d=96, rot=24, T=509, interleaved=True, norm=False, spread=1),
        # a long prompt: as much data as a copy of 512 MB moves; frequencies scaled for a long context
        _rope("rope_long", n=2, heads=32, d=128, rot=128, T=8192, scaled=8.0, start=100000),
        # training steps: keys of a small batch of odd length, queries of a large one
        _rope("rope_train_odd", n=6, heads=8, d=64, rot=64, T=333, backward=True),
        _rope("rope_train", n=8, heads=16, d=128, rot=128, T=2048, interleaved=True, backward=True),
        # ---- attention to another sequence's states ----
        # one token for each of 4 sequences over an encoder's 1500 states: latency
        _attention("attention_token", n=4, heads=16, kv_heads=16, d=64, Tq=1, Tk=1500, ragged=True),
        # one token over long memories with shared heads: reading the states
        _attention("attention_token_long", n=4, heads=32, kv_heads=8, d=128, Tq=1, Tk=32768, ragged=True),
        # a feature map's 32 x 32 pixels to a short text, heads of 40 channels
        _attention("attention_map", n=8, heads=8, kv_heads=8, d=40, Tq=1024, Tk=77),
        # a decoder's prompt over an encoder's states
        _attention("attention_prompt", n=8, heads=16, kv_heads=16, d=64, Tq=448, Tk=1500, ragged=True),
        # long sequences, shared heads: the matrix units
        _attention("attention_long", n=1, heads=32, kv_heads=8, d=128, Tq=4096, Tk=4096),
        # training steps: odd lengths, and the largest product
        _attention("attention_train_odd", n=4, heads=8, kv_heads=8, d=64, Tq=300, Tk=213, ragged=True, backward=True),
        _attention("attention_train", n=2, heads=16, kv_heads=4, d=128, Tq=2048, Tk=2048, backward=True),
    ]


def _rope(name=None, n=1, heads=1, d=64, rot=64, T=1, interleaved=False, norm=True, start=0, spread=0, scaled=1.0, backward=False):
    case = {"name": name, "op": "head_rope", "n": n, "heads": heads, "d": d, "rot": rot, "T": T, "interleaved": interleaved,
            "norm": norm, "start": start, "spread": bool(spread), "scaled": scaled, "backward": backward}
    return case if name else {k: v for k, v in case.items() if k != "name"}


def _attention(name=None, n=1, heads=1, kv_heads=1, d=64, Tq=1, Tk=1, ragged=False, backward=False):
    case = {"name": name, "op": "attention", "n": n, "heads": heads, "kv_heads": kv_heads, "d": d, "Tq": Tq, "Tk": Tk,
            "ragged": ragged, "backward": backward}
    return case if name else {k: v for k, v in case.items() if k != "name"}


MOST_ROPE_VALUES = 1 << 26                      # of one tensor
MOST_ATTENTION_FLOPS = 1.35e11                  # of one of the products
MOST_STATES = 1 << 27                           # values of k and of v


def _spread(rng, lo, hi):
    """A whole number from lo to hi, uniform in its logarithm."""
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random() + 0.5)))


def draw(rng):
    d = rng.choice([16, 32, 40, 64, 64, 72, 80, 96, 128, 128])
    n = _spread(rng, 1, 16)
    if rng.random() < 0.42:
        heads = _spread(rng, 1, 40)
        T = 1 if rng.random() < 0.2 else _spread(rng, 2, 8192)
        T = max(1, min(T, MOST_ROPE_VALUES // (n * heads * d)))
        rot = rng.choice([d, d, d // 2, d // 4 * 2 or 2])
        return _rope(None, n, heads, d, rot, T, rng.random() < 0.5, rng.random() < 0.7, rng.choice([0, 0, 1000, 200000]), rng.random() < 0.5,
                     rng.choice([1.0, 4.0, 8.0]), rng.random() < 0.4)
    kv_heads = _spread(rng, 1, 16)
    heads = kv_heads * rng.choice([1, 1, 1, 2, 4, 8])
    backward = rng.random() < 0.4
    Tk = _spread(rng, 1, 8192 if backward else 32768)
    Tq = 1 if not backward and rng.random() < 0.35 else _spread(rng, 2, 4096)
    Tk = max(1, min(Tk, MOST_STATES // (2 if backward else 1) // (n * kv_heads * d)))
    most = MOST_ATTENTION_FLOPS / (4 if backward else 1)
    Tq = max(1, min(Tq, int(most / (2.0 * n * heads * Tk * d)), MOST_STATES // 4 // (n * heads * d) or 1, (1 << 30) // (n * heads * Tk) or 1))
    return _attention(None, n, heads, kv_heads, d, Tq, Tk, rng.random() < 0.5, backward)


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _frequencies(case):
    """One angle a position for each pair; scaled: the base raised so that a context of `scaled` times the length is spanned."""
    rot = case["rot"]
    base = 10000.0 * (case["scaled"] ** (rot / (rot - 2.0)) if rot > 2 else 1.0)
    return (base ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)).astype(np.float32)


def _inputs(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    n, d = case["n"], case["d"]
    if case["op"] == "head_rope":
        H, T = case["heads"], case["T"]
        at = case["start"] + torch.arange(T, device=DEVICE, dtype=torch.float64)
        first = torch.randint(0, 1000, (n if case["spread"] else 1, 1), generator=g, device=DEVICE)    # sequences of different age
        s = {"x": normal(n, H * d, 1, T) * 2.0, "positions": (at + first).float().view(-1, 1, 1, T).contiguous(),
             "frequencies": torch.from_numpy(_frequencies(case)).to(DEVICE),
             "gamma": 0.8 + 0.4 * torch.rand(d, generator=g, device=DEVICE)}
        if case["backward"]:
            s["dy"] = normal(n, H * d, 1, T) * 1e-3                  # gradients are small
        return s
    H, Hk, Tq, Tk = case["heads"], case["kv_heads"], case["Tq"], case["Tk"]
    s = {"q": normal(n, H * d, 1, Tq), "k": normal(n, Hk * d, 1, Tk), "v": normal(n, Hk * d, 1, Tk)}
    if case["ragged"]:
        lengths = torch.randint(Tk // 2, Tk + 1, (n,), generator=g, device=DEVICE)
        lengths[0] = Tk                                              # the longest sequence gives the batch its extent
        if n > 1:
            lengths[n - 1] = 0                                       # a sequence without any state
        s["lengths"] = lengths.float().view(n, 1, 1, 1)
    if case["backward"]:
        s["dy"] = normal(n, H * d, 1, Tq) * 1e-3
    return s


@dataclasses.dataclass
class State:
    case: dict
    inputs: dict                  # the plain form's
    runner: object = None         # the framework's captured graph, its inputs in place
    results: dict = None          # the graph's tensors that a pass answers with


def prepare(case, seed):
    state = State(case, _inputs(case, seed))
    if own:
        state.runner, state.results = _captured(case, state.inputs)
        state.inputs = None                                          # they are in the graph's arena
    return state


def run(state):
    if own:
        state.runner.replay()
        return state.results
    case, s = state.case, state.inputs
    if case["op"] == "head_rope":
        return _plain_rope(case, **s)
    return _plain_attention(case, **s)


# ---- the framework's calls ---------------------------------------------------------------------------------------------------

_origin = []


def _captured(case, s):
    import workloads
    from paper_2012_02732_amd import GraphRunner
    nodes, inputs = [], {}

    def given(name):
        t = s[name]
        inputs[len(nodes)] = t
        nodes.append(workloads.Node("input", [], dict(zip("nchw", t.shape)), [], tuple(t.shape)))
        return len(nodes) - 1

    def node(op, preds, shape, weights=(), shared=(), **params):
        nodes.append(workloads.Node(op, list(preds), params, list(weights), tuple(shape), 1.0, list(shared)))
        return len(nodes) - 1

    out, d = {}, case["d"]
    if case["op"] == "head_rope":
        x, pos = given("x"), given("positions")
        weights = [s["frequencies"].cpu().numpy()] + ([s["gamma"].cpu().numpy()] if case["norm"] else [])
        how = dict(heads=case["heads"], rot=case["rot"], interleaved=int(case["interleaved"]), eps=EPS, factor=1.0)
        y = out["y"] = node("head_rope", [x, pos], s["x"].shape, weights, **how)
        if case["backward"]:
            dy, shared = given("dy"), [(y, j) for j in range(len(weights))]
            out["dx"] = node("head_rope_dgrad", [dy, x, pos], s["x"].shape, shared=shared, **how)
            if case["norm"]:
                out["dgamma"] = node("head_rope_wgrad", [dy, x, pos], (1, d, 1, 1), shared=shared, **how)
    else:
        q, k, v = given("q"), given("k"), given("v")
        lengths = [given("lengths")] if case["ragged"] else []
        how = dict(heads=case["heads"], kv_heads=case["kv_heads"], scale=d ** -0.5)
        y = out["y"] = node("attention", [q, k, v] + lengths, s["q"].shape, **how)
        if case["backward"]:
            dy = given("dy")
            rows = node("attention_rows", [dy, y], (case["n"], 3 * case["heads"], 1, case["Tq"]), heads=case["heads"])
            for name, of in (("dq", "q"), ("dk", "k"), ("dv", "v")):
                out[name] = node("attention_" + name, [dy, rows, q, k, v] + lengths, s[of].shape, **how)
    if not _origin:
        _origin.append(torch.cuda.Stream(DEVICE))
    w = workloads.Workload("operator", nodes, inputs[0], sorted(out.values()), inputs=inputs)
    r = GraphRunner(w, DEVICE)
    r.prepare(plan_trials=1, origin_stream=_origin[0].cuda_stream)   # one stream for all graphs of this program: passes follow each other
    return r, {name: r.tensor(i) for name, i in out.items()}


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _pairs(case, t):
    """First and second elements of the rotated pairs, and the channels behind them, of [n][H][d][T]."""
    rot = case["rot"]
    if case["interleaved"]:
        return t[:, :, 0:rot:2], t[:, :, 1:rot:2], t[:, :, rot:]
    return t[:, :, :rot // 2], t[:, :, rot // 2:rot], t[:, :, rot:]


def _joined(case, a, b, rest):
    if case["interleaved"]:
        return torch.cat([torch.stack([a, b], 3).flatten(2, 3), rest], 2)
    return torch.cat([a, b, rest], 2)


def _plain_rope(case, x, positions, frequencies, gamma, dy=None):
    n, H, d, T = case["n"], case["heads"], case["d"], case["T"]
    angle = positions.view(-1, 1, 1, T).double() * frequencies.double().view(1, 1, -1, 1)     # far positions: 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    x = x.view(n, H, d, T)
    gamma = gamma.view(1, 1, d, 1)
    if case["norm"]:
        r = torch.rsqrt((x * x).mean(2, keepdim=True) + EPS)
        u = x * r * gamma
    else:
        u = x
    a, b, rest = _pairs(case, u)
    out = {"y": _joined(case, a * cos - b * sin, a * sin + b * cos, rest).view(n, H * d, 1, T)}
    if case["backward"]:
        a, b, rest = _pairs(case, dy.view(n, H, d, T))
        du = _joined(case, a * cos + b * sin, b * cos - a * sin, rest)
        if case["norm"]:
            xh = x * r
            out["dgamma"] = (du * xh).sum((0, 1, 3)).view(1, d, 1, 1)
            du = du * gamma
            du = r * (du - xh * (du * xh).mean(2, keepdim=True))
        out["dx"] = du.reshape(n, H * d, 1, T)
    return out


def _plain_attention(case, q, k, v, lengths=None, dy=None):
    n, H, Hk, d, Tq, Tk = (case[x] for x in ("n", "heads", "kv_heads", "d", "Tq", "Tk"))
    G, scale = H // Hk, d ** -0.5
    q = q.view(n, Hk, G, d, Tq)
    k, v = k.view(n, Hk, 1, d, Tk), v.view(n, Hk, 1, d, Tk)
    score = torch.matmul(q.transpose(3, 4), k) * scale                                       # [n][Hk][G][Tq][Tk]
    if lengths is not None:
        hidden = torch.arange(Tk, device=q.device).view(1, 1, 1, 1, Tk) >= lengths.view(n, 1, 1, 1, 1)
        score = score.masked_fill(hidden, -math.inf)
        top = score.amax(4, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)                                        # rows without a key
    else:
        top = score.amax(4, keepdim=True)
    p = torch.exp(score - top)
    del score
    total = p.sum(4, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    y = torch.matmul(v, p.transpose(3, 4))                                                   # [n][Hk][G][d][Tq]
    out = {"y": y.reshape(n, H * d, 1, Tq)}
    if case["backward"]:
        g = dy.view(n, Hk, G, d, Tq)
        out["dv"] = torch.matmul(g, p).sum(2).view(n, Hk * d, 1, Tk)
        ds = torch.matmul(g.transpose(3, 4), v)
        ds = p * (ds - (g * y).sum(3).unsqueeze(4)) * scale
        del p
        out["dq"] = torch.matmul(k, ds.transpose(3, 4)).reshape(n, H * d, 1, Tq)
        out["dk"] = torch.matmul(q, ds).sum(2).view(n, Hk * d, 1, Tk)
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = {name: t.double() for name, t in _inputs(case, seed).items()}
    leaves = {}

    def leaf(name):
        leaves[name] = s[name].requires_grad_(case["backward"])
        return leaves[name]

    n, H, d = case["n"], case["heads"], case["d"]
    with torch.set_grad_enabled(case["backward"]):
        if case["op"] == "head_rope":
            T, rot = case["T"], case["rot"]
            u = leaf("x").reshape(n * H, d, T)
            if case["norm"]:
                u = u / (u.square().sum(1, keepdim=True) / d + EPS).sqrt() * leaf("gamma")[None, :, None]
            turned = u[:, :rot].reshape(n * H, rot // 2, 2, T).transpose(1, 2) if case["interleaved"] else u[:, :rot].reshape(n * H, 2, rot // 2, T)
            angle = s["positions"].reshape(-1, 1, T) * s["frequencies"][None, :, None]       # [1 or n][rot / 2][T]
            angle = angle.expand(n, rot // 2, T).repeat_interleave(H, 0)
            z = torch.complex(turned[:, 0], turned[:, 1]) * torch.polar(torch.ones_like(angle), angle)
            turned = torch.stack([z.real, z.imag], 2 if case["interleaved"] else 1).reshape(n * H, rot, T)
            y = torch.cat([turned, u[:, rot:]], 1).reshape(n, H * d, 1, T)
            names = {"x": "dx", "gamma": "dgamma"}
        else:
            Hk, Tq, Tk = case["kv_heads"], case["Tq"], case["Tk"]
            if n * H * float(Tq) * Tk > 2 ** 30:
                return None
            q, k, v = leaf("q"), leaf("k"), leaf("v")
            images = []
            for i in range(n):                                       # an image at a time, over the keys that it has
                L = int(s["lengths"][i]) if case["ragged"] else Tk
                if L == 0:
                    images.append(torch.zeros(H * d, 1, Tq, dtype=torch.float64, device=DEVICE) * q[i])
                    continue
                qi = q[i].view(H, d, Tq)
                ki, vi = (t[i].view(Hk, d, Tk)[:, :, :L].repeat_interleave(H // Hk, 0) for t in (k, v))
                w = torch.softmax(torch.bmm(qi.transpose(1, 2), ki) / math.sqrt(d), 2)
                images.append(torch.bmm(w, vi.transpose(1, 2)).transpose(1, 2).reshape(H * d, 1, Tq))
            y = torch.stack(images)
            names = {"q": "dq", "k": "dk", "v": "dv"}
        out = {"y": y.detach()}
        if case["backward"]:
            found = torch.autograd.grad(y, list(leaves.values()), s["dy"], allow_unused=True)
            for name, t in zip(leaves, found):
                out[names[name]] = t if name != "gamma" else t.view(1, d, 1, 1)
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------

def work(case):
    """Every input read once, every result written once; the products of the attention and of its gradients (two forward, dP, dV,
    dQ and dK backward) over all keys there can be."""
    n, d = float(case["n"]), case["d"]
    if case["op"] == "head_rope":
        x = n * case["heads"] * d * case["T"]
        positions = (n if case["spread"] else 1) * case["T"]
        tensors = 4 if case["backward"] else 2
        return {"bytes": 4 * (tensors * x + positions + case["rot"] / 2 + d), "flops": x * (20 if case["backward"] else 7)}
    queries, states = n * case["heads"] * d * case["Tq"], n * case["kv_heads"] * d * case["Tk"]
    values = (2 * queries + 2 * states) * (2 if case["backward"] else 1)
    product = 2.0 * queries * case["Tk"]
    return {"bytes": 4 * values, "flops": product * (6 if case["backward"] else 2)}
