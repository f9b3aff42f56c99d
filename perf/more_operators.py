"""Operators of a transformer block that is trained, as timed cases: the norm of a token's channels, dropout, and attention with a learned
bias of the distance between tokens.

Tensors are fp32 and channel-major, as the 1 x 1 convolutions around these operators leave and take them: [n][c][1][T], the T tokens of
an image (a sequence) contiguous. Each operator is a node of a graph (position bias and attention with it: two):

layer norm           x [n][c][1][T], gamma[c], beta[c]: y = gamma (x - mean) / sqrt(variance + eps) + beta, over the c channels of a token
layer norm backward  dx, and dgamma and dbeta as [2][c][1][1], from dy
dropout              x of any shape, a seed of 64 bits in the bit patterns of two values, and a residual or none:
                       y = residual + (kept ? x / (1 - rate) : 0)
                     Element e is kept if word e % 4 of Philox4x32-10 (counter e / 4 in two words, the site, 0; key: the seed) is at least
                     rate 2^32. The gradient is the same operator on dy
position bias        table [buckets][heads] -> [1][heads][1][2 m + 1]: the bias of distance d = -m .. m (m: the largest distance told apart)
                     With b = buckets / 2 for each direction (keys behind the query: the upper half), or b = buckets for keys up to
                     the query alone (keys behind it: minus infinity, they are not seen), and exact = b / 2:
                       bucket(d) = |d| below exact, else min(b - 1, exact + floor((b - exact) log(|d| / exact) / log(m / exact)))
biased attention     q [n][H d][1][Tq], k, v [n][Hk d][1][Tk], lengths [n], bias: p[i][j] = softmax over j < lengths[image] of
                       scale <q_i, k_j> + bias[head][j - i - offset], distances beyond m as m; offset 0 ("first"), or the keys that count
                       less Tq ("last": the queries are the last tokens). y_i = sum_j p[i][j] v_j; without a key that is seen: 0
its backward         dq, dk, dv and dtable from dy

A pass of a training case is the forward operator and its gradients, as one graph. The framework's side keeps a captured graph whose
inputs lie in its arena, as every program of this framework does, and replays it.
"""
import dataclasses
import math

import numpy as np
import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5


def listed():
    return [
        # ---- layer norm ----
        # one new token for each of 8 sequences: the smallest call, all of it latency
        _norm("norm_token", n=8, c=1024, T=1),
        # a long prompt through a wide network: as much data as a copy of 512 MB moves
        _norm("norm_long", n=2, c=4096, T=8192),
        # training steps: a small batch of odd length, and a large one
        _norm("norm_train_odd", n=6, c=520, T=333, backward=True),
        _norm("norm_train", n=8, c=1024, T=4096, backward=True),
        # ---- dropout ----
        # the end of a small network: an odd number of values, no residual
        _dropout("dropout_odd", n=3, c=511, T=77, rate=0.5),
        # a block's second half in a training step: residual sum, and the gradient with the same mask
        _dropout("dropout_train_odd", n=6, c=520, T=333, rate=0.1, residual=True, backward=True),
        _dropout("dropout_train", n=8, c=1024, T=8192, rate=0.1, residual=True, backward=True),
        # ---- attention with a learned bias of distances ----
        # one new token for each of 4 sequences, the last of the keys that count: latency
        _attention("bias_token", n=4, heads=16, kv_heads=16, d=64, Tq=1, Tk=1500, ragged=True, at="last"),
        # an encoder's sequences of different lengths, both directions
        _attention("bias_encoder", n=8, heads=16, kv_heads=16, d=64, Tq=512, Tk=512, ragged=True),
        # a long prompt that only looks back, shared heads
        _attention("bias_long", n=1, heads=32, kv_heads=8, d=128, Tq=4096, Tk=4096, both=False),
        # training steps: odd lengths, and a large product
        _attention("bias_train_odd", n=4, heads=8, kv_heads=8, d=64, Tq=300, Tk=213, ragged=True, backward=True),
        _attention("bias_train", n=2, heads=16, kv_heads=16, d=64, Tq=2048, Tk=2048, backward=True),
    ]


def _case(name, op, **sizes):
    return {**({"name": name} if name else {}), "op": op, **sizes}


def _norm(name=None, n=1, c=1, T=1, backward=False):
    return _case(name, "layer_norm", n=n, c=c, T=T, backward=backward)


def _dropout(name=None, n=1, c=1, T=1, rate=0.1, residual=False, backward=False):
    return _case(name, "dropout", n=n, c=c, T=T, rate=rate, residual=residual, backward=backward)


def _attention(name=None, n=1, heads=1, kv_heads=1, d=64, Tq=1, Tk=1, ragged=False, backward=False, buckets=32, largest=128, both=True, at="first"):
    return _case(name, "attention", n=n, heads=heads, kv_heads=kv_heads, d=d, Tq=Tq, Tk=Tk, ragged=ragged, backward=backward,
                 buckets=buckets, largest=largest, both=both, at=at)


MOST_VALUES = 1 << 26                           # of one tensor of norm or dropout
MOST_ATTENTION_FLOPS = 1.35e11                  # of one of the products
MOST_STATES = 1 << 26                           # values of k and of v


def _spread(rng, lo, hi):
    """A whole number from lo to hi, uniform in its logarithm."""
    return max(lo, min(hi, int(lo * (hi / lo) ** rng.random() + 0.5)))


def draw(rng):
    which = rng.random()
    n = _spread(rng, 1, 16)
    if which < 0.5:
        c = _spread(rng, 8, 4096)
        T = 1 if rng.random() < 0.2 else _spread(rng, 2, 8192)
        T = max(1, min(T, MOST_VALUES // (n * c)))
        if which < 0.3:
            return _norm(None, n, c, T, rng.random() < 0.5)
        return _dropout(None, n, c, T, rng.choice([0.05, 0.1, 0.1, 0.25, 0.5]), rng.random() < 0.6, rng.random() < 0.5)
    d = rng.choice([16, 32, 40, 64, 64, 72, 80, 96, 128])
    kv_heads = _spread(rng, 1, 16)
    heads = kv_heads * rng.choice([1, 1, 1, 2, 4])
    backward = rng.random() < 0.4
    Tk = _spread(rng, 2, 4096) if backward else _spread(rng, 1, 16384)
    Tq = 1 if not backward and rng.random() < 0.35 else _spread(rng, 2, 4096)
    Tk = max(1, min(Tk, MOST_STATES // (2 if backward else 1) // (n * kv_heads * d)))
    most = MOST_ATTENTION_FLOPS / (4 if backward else 1)
    Tq = max(1, min(Tq, int(most / (2.0 * n * heads * Tk * d)), MOST_STATES // 2 // (n * heads * d) or 1, (1 << 28 if not backward else 1 << 27) // (n * heads * Tk) or 1))
    buckets, largest = rng.choice([(32, 128), (32, 128), (16, 40), (64, 500), (8, 10)])
    return _attention(None, n, heads, kv_heads, d, Tq, Tk, rng.random() < 0.5, backward, buckets, largest, rng.random() < 0.5,
                      rng.choice(["first", "last"]) if Tq > 1 else "last")


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _inputs(case, seed):
    g = torch.Generator(DEVICE).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEVICE)

    n = case["n"]
    if case["op"] == "attention":
        H, Hk, d, Tq, Tk = (case[x] for x in ("heads", "kv_heads", "d", "Tq", "Tk"))
        s = {"q": normal(n, H * d, 1, Tq), "k": normal(n, Hk * d, 1, Tk), "v": normal(n, Hk * d, 1, Tk), "table": normal(case["buckets"], H) * 2.0}
        if case["ragged"]:
            lengths = torch.randint(Tk // 2, Tk + 1, (n,), generator=g, device=DEVICE)
            lengths[0] = Tk                                          # the longest sequence gives the batch its extent
            if n > 1:
                lengths[n - 1] = 0                                   # a sequence without any state
            s["lengths"] = lengths.float().view(n, 1, 1, 1)
        if case["backward"]:
            s["dy"] = normal(n, H * d, 1, Tq) * 1e-3                 # gradients are small
        return s
    c, T = case["c"], case["T"]
    x = normal(n, c, 1, T)
    if case["op"] == "layer_norm":                                   # channels of a network's residual sum have different means and spreads
        s = {"x": x * (0.5 + 3.0 * torch.rand(1, c, 1, 1, generator=g, device=DEVICE)) + normal(1, c, 1, 1),
             "gamma": 0.8 + 0.4 * torch.rand(c, generator=g, device=DEVICE), "beta": normal(c) * 0.1}
    else:
        s = {"x": x, "seed": torch.randint(-2 ** 31, 2 ** 31, (1, 1, 1, 2), generator=g, device=DEVICE).to(torch.int32).view(torch.float32)}
        if case["residual"]:
            s["residual"] = normal(n, c, 1, T) * 2.0
    if case["backward"]:
        s["dy"] = normal(n, c, 1, T) * 1e-3
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
    return {"layer_norm": _plain_norm, "dropout": _plain_dropout, "attention": _plain_attention}[state.case["op"]](state.case, **state.inputs)


# ---- the framework's calls ---------------------------------------------------------------------------------------------------

_origin = []
SITE = 7                                        # which dropout of a network: each has a mask of its own


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
        nodes.append(workloads.Node(op, list(preds), params, [w.cpu().numpy() for w in weights], tuple(shape), 1.0, list(shared)))
        return len(nodes) - 1

    out = {}
    if case["op"] == "layer_norm":
        x = given("x")
        y = out["y"] = node("layer_norm", [x], s["x"].shape, [s["gamma"], s["beta"]], eps=EPS)
        if case["backward"]:
            dy, shared = given("dy"), [(y, 0), (y, 1)]
            out["dx"] = node("layer_norm_dgrad", [dy, x], s["x"].shape, shared=shared, eps=EPS)
            out["dweights"] = node("layer_norm_wgrad", [dy, x], (2, case["c"], 1, 1), shared=shared, eps=EPS)
    elif case["op"] == "dropout":
        x, seed = given("x"), given("seed")
        how = dict(rate=case["rate"], site=SITE)
        out["y"] = node("dropout", [x, seed] + ([given("residual")] if case["residual"] else []), s["x"].shape, **how)
        if case["backward"]:
            out["dx"] = node("dropout", [given("dy"), seed], s["x"].shape, **how)
    else:
        q, k, v = given("q"), given("k"), given("v")
        lengths = [given("lengths")] if case["ragged"] else []
        spans = dict(heads=case["heads"], buckets=case["buckets"], max_distance=case["largest"], both=int(case["both"]))
        distances = (1, case["heads"], 1, 2 * case["largest"] + 1)
        bias = node("position_bias", [], distances, [s["table"]], **spans)
        how = dict(heads=case["heads"], kv_heads=case["kv_heads"], scale=case["d"] ** -0.5, bias=case["at"])
        y = out["y"] = node("attention", [q, k, v] + lengths + [bias], s["q"].shape, **how)
        if case["backward"]:
            dy = given("dy")
            rows = node("attention_rows", [dy, y], (case["n"], 3 * case["heads"], 1, case["Tq"]), heads=case["heads"])
            read = [dy, rows, q, k, v] + lengths + [bias]
            for name, of in (("dq", "q"), ("dk", "k"), ("dv", "v")):
                out[name] = node("attention_" + name, read, s[of].shape, **how)
            dbias = node("attention_dbias", read, distances, **how)
            out["dtable"] = node("position_bias_wgrad", [dbias], (case["buckets"], case["heads"], 1, 1), **spans)
    if not _origin:
        _origin.append(torch.cuda.Stream(DEVICE))
    w = workloads.Workload("operator", nodes, inputs[0], sorted(out.values()), inputs=inputs)
    r = GraphRunner(w, DEVICE)
    r.prepare(plan_trials=1, origin_stream=_origin[0].cuda_stream)   # one stream for all graphs of this program: passes follow each other
    return r, {name: r.tensor(i) for name, i in out.items()}


# ---- the plain forms ---------------------------------------------------------------------------------------------------------

def _plain_norm(case, x, gamma, beta, dy=None):
    c = case["c"]
    g, b = gamma.view(1, c, 1, 1), beta.view(1, c, 1, 1)
    centred = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((centred * centred).mean(1, keepdim=True) + EPS)
    xh = centred * r
    out = {"y": xh * g + b}
    if case["backward"]:
        u = dy * g
        out["dx"] = r * (u - u.mean(1, keepdim=True) - xh * (u * xh).mean(1, keepdim=True))
        out["dweights"] = torch.stack([(dy * xh).sum((0, 2, 3)), dy.sum((0, 2, 3))]).view(2, c, 1, 1)
    return out


WORD = 0xFFFFFFFF


def _philox(block, site, key0, key1):
    """The four words of each block, [blocks][4], in integers of 64 bits."""
    words = [block & WORD, block >> 32, torch.full_like(block, site), torch.zeros_like(block)]
    for _ in range(10):
        a, b = words[0] * 0xD2511F53, words[2] * 0xCD9E8D57          # (modulo 2^64: both halves are there)
        words = [((b >> 32) & WORD) ^ words[1] ^ key0, b & WORD, ((a >> 32) & WORD) ^ words[3] ^ key1, a & WORD]
        key0, key1 = (key0 + 0x9E3779B9) & WORD, (key1 + 0xBB67AE85) & WORD
    return torch.stack(words, 1)


def _plain_dropout(case, x, seed, residual=None, dy=None):
    values = x.numel()
    key = seed.view(torch.int32).flatten().long() & WORD             # (0-d tensors: nothing goes to the host)
    words = _philox(torch.arange((values + 3) // 4, device=x.device), SITE, key[0], key[1])
    limit = round(float(np.float32(case["rate"])) * 2.0 ** 32)
    kept = (words.flatten()[:values] >= limit).view(x.shape)
    scale = 2.0 ** 32 / (2.0 ** 32 - limit)
    y = torch.where(kept, x * scale, 0.0)
    out = {"y": y if residual is None else residual + y}
    if case["backward"]:
        out["dx"] = torch.where(kept, dy * scale, 0.0)
    return out


def _bucket(case, distance):
    """Of whole distances, logarithms in 64 bits; a border counts as reached from 1e-9 below it on."""
    b = case["buckets"] // 2 if case["both"] else case["buckets"]
    exact = b // 2
    far = distance.abs()
    log = torch.log(far.clamp(min=1).double() / exact) / math.log(case["largest"] / exact) * (b - exact)
    far = torch.where(far < exact, far, (exact + torch.floor(log + 1e-9).long()).clamp(max=b - 1))
    return far + (distance > 0).long() * b if case["both"] else far


def _plain_attention(case, q, k, v, table, lengths=None, dy=None):
    n, H, Hk, d, Tq, Tk = (case[x] for x in ("n", "heads", "kv_heads", "d", "Tq", "Tk"))
    G, scale, m = H // Hk, d ** -0.5, case["largest"]
    distance = torch.arange(-m, m + 1, device=q.device)
    bucket = _bucket(case, distance)
    bias = table[bucket]                                                                     # [2 m + 1][H]
    if not case["both"]:
        bias = bias.masked_fill((distance > 0).view(-1, 1), -math.inf)
    keys = torch.full((n,), Tk, device=q.device) if lengths is None else lengths.view(n).long()
    first = torch.zeros_like(keys) if case["at"] == "first" else keys - Tq
    at = torch.arange(Tk, device=q.device).view(1, 1, Tk) - torch.arange(Tq, device=q.device).view(1, Tq, 1) - first.view(n, 1, 1)
    at = at.clamp(-m, m) + m                                                                 # [n][Tq][Tk]
    hidden = torch.arange(Tk, device=q.device).view(1, 1, 1, Tk) >= keys.view(n, 1, 1, 1)
    q = q.view(n, Hk, G, d, Tq)
    k, v = k.view(n, Hk, 1, d, Tk), v.view(n, Hk, 1, d, Tk)
    score = torch.matmul(q.transpose(3, 4), k) * scale                                       # [n][Hk][G][Tq][Tk]
    score = score + bias.t().contiguous()[:, at].transpose(0, 1).reshape(score.shape)
    p = score.masked_fill(hidden.unsqueeze(1), -math.inf)
    del score
    top = p.amax(4, keepdim=True)
    p = torch.exp(p - torch.where(top == -math.inf, 0.0, top))                               # rows without a key: 0
    total = p.sum(4, keepdim=True)
    p = p / torch.where(total == 0, 1.0, total)
    y = torch.matmul(v, p.transpose(3, 4))                                                   # [n][Hk][G][d][Tq]
    out = {"y": y.reshape(n, H * d, 1, Tq)}
    if case["backward"]:
        g = dy.view(n, Hk, G, d, Tq)
        out["dv"] = torch.matmul(g, p).sum(2).view(n, Hk * d, 1, Tk)
        ds = torch.matmul(g.transpose(3, 4), v)
        ds = p * (ds - (g * y).sum(3).unsqueeze(4))
        del p
        # Sums along the diagonals: with rows of Tq + Tk - 1 in the place of Tq + Tk values, row Tq - 1 - i begins i columns further on.
        backwards = torch.arange(Tq - 1, -1, -1, device=q.device)
        by_distance = torch.zeros(2 * m + 1, H, device=q.device, dtype=torch.float64)        # millions of terms of both signs
        for image in range(n):
            wide = torch.cat([ds[image].flatten(0, 1)[:, backwards], torch.zeros(H, Tq, Tq, device=q.device)], 2)
            sheared = wide.flatten(1)[:, :Tq * (Tq + Tk - 1)].view(H, Tq, Tq + Tk - 1)
            reached = torch.arange(Tq + Tk - 1, device=q.device) - (Tq - 1) - first[image]   # j - i - offset
            by_distance.index_add_(0, reached.clamp(-m, m) + m, sheared.sum(1, dtype=torch.float64).t())
        dtable = torch.zeros(case["buckets"], H, device=q.device, dtype=torch.float64).index_add_(0, bucket, by_distance)
        out["dtable"] = dtable.float().view(case["buckets"], H, 1, 1)
        ds = ds * scale
        out["dq"] = torch.matmul(k, ds.transpose(3, 4)).reshape(n, H * d, 1, Tq)
        out["dk"] = torch.matmul(q, ds).sum(2).view(n, Hk * d, 1, Tk)
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    return {"layer_norm": _exact_norm, "dropout": _exact_dropout, "attention": _exact_attention}[case["op"]](case, s)


def _exact_norm(case, s):
    x, gamma, beta = (s[name].double().requires_grad_(case["backward"]) for name in ("x", "gamma", "beta"))
    with torch.set_grad_enabled(case["backward"]):
        tokens = x[:, :, 0].transpose(1, 2)                          # [n][T][c]
        variance, mean = torch.var_mean(tokens, 2, unbiased=False, keepdim=True)
        y = ((tokens - mean) / (variance + EPS).sqrt() * gamma + beta).transpose(1, 2).unsqueeze(2)
    out = {"y": y.detach()}
    if case["backward"]:
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), s["dy"].double())
        out["dx"], out["dweights"] = dx, torch.stack([dgamma, dbeta]).view(2, -1, 1, 1)
    return out


def _exact_dropout(case, s):
    def product(a, b):                                               # of a number and a constant of 32 bits: high and low word, from halves of 16 bits
        low, high = a & 0xFFFF, a >> 16
        x, y = low * b, high * b                                     # below 2^48
        total = x + ((y & 0xFFFF) << 16)
        return (y >> 16) + (total >> 32), total & WORD

    values = s["x"].numel()
    key = [int(v) & WORD for v in s["seed"].view(torch.int32).flatten().tolist()]
    e = torch.arange((values + 3) // 4, device=DEVICE)
    left, right = (e & WORD, torch.full_like(e, SITE)), (e >> 32, torch.zeros_like(e))       # words 0 and 2, 1 and 3
    for turn in range(10):
        k0, k1 = (key[0] + turn * 0x9E3779B9) & WORD, (key[1] + turn * 0xBB67AE85) & WORD
        h0, l0 = product(left[0], 0xD2511F53)
        h1, l1 = product(left[1], 0xCD9E8D57)
        left, right = (h1 ^ right[0] ^ k0, h0 ^ right[1] ^ k1), (l1, l0)
    kept = torch.empty(len(e), 4, dtype=torch.bool, device=DEVICE)
    limit = int(np.rint(np.float64(np.float32(case["rate"])) * 4294967296.0))
    for j, w in enumerate((left[0], right[0], left[1], right[1])):
        kept[:, j] = w >= limit
    kept = kept.view(-1)[:values].view(s["x"].shape)
    keep = 1.0 - limit / 4294967296.0

    def masked(t):
        return torch.where(kept, t.double() / keep, torch.zeros((), dtype=torch.float64, device=DEVICE))

    out = {"y": masked(s["x"])}
    if case["residual"]:
        out["y"] = out["y"] + s["residual"].double()
    if case["backward"]:
        out["dx"] = masked(s["dy"])
    return out


def _exact_buckets(case):
    """Bucket of each distance 0 .. m, in whole numbers: step j is reached where (d / exact)^steps >= (m / exact)^j."""
    b = case["buckets"] // 2 if case["both"] else case["buckets"]
    exact, m = b // 2, case["largest"]
    steps, found = b - exact, []
    for d in range(m + 1):
        j = d - exact if d < exact else max(j for j in range(steps + 1) if d ** steps * exact ** j >= m ** j * exact ** steps)
        found.append(min(exact + j, b - 1))
    return b, found


def _exact_attention(case, s):
    n, H, Hk, d, Tq, Tk, m = (case[x] for x in ("n", "heads", "kv_heads", "d", "Tq", "Tk", "largest"))
    if n * H * float(Tq) * Tk > 2 ** 30:
        return None
    b, near = _exact_buckets(case)
    near = torch.tensor(near, device=DEVICE)
    q, k, v, table = (s[name].double().requires_grad_(case["backward"]) for name in ("q", "k", "v", "table"))
    with torch.set_grad_enabled(case["backward"]):
        images = []
        for i in range(n):                                           # an image and a head at a time, over the keys that it has
            L = int(s["lengths"][i]) if case["ragged"] else Tk
            if L == 0:
                images.append(torch.zeros(H * d, 1, Tq, dtype=torch.float64, device=DEVICE) * q[i])
                continue
            first = L - Tq if case["at"] == "last" else 0
            away = torch.arange(L, device=DEVICE)[None, :] - (torch.arange(Tq, device=DEVICE)[:, None] + first)
            row = near[away.abs().clamp(max=m)] + (b * (away > 0) if case["both"] else 0)
            hidden = away > (Tk + Tq if case["both"] else 0)
            seen = ~hidden.all(1, keepdim=True)
            heads = []
            for h in range(H):
                qh, kh, vh = q[i].view(H, d, Tq)[h], k[i].view(Hk, d, Tk)[h * Hk // H, :, :L], v[i].view(Hk, d, Tk)[h * Hk // H, :, :L]
                score = torch.mm(qh.t().contiguous(), kh.contiguous()) / math.sqrt(d) + table[:, h][row]
                w = torch.softmax(score.masked_fill(hidden & seen, -math.inf), 1) * seen
                heads.append(torch.mm(vh.contiguous(), w.t().contiguous()))
            images.append(torch.stack(heads).view(H * d, 1, Tq))
        y = torch.stack(images)
    out = {"y": y.detach()}
    if case["backward"]:
        out["dv"], dtable, out["dq"], out["dk"] = torch.autograd.grad(y, (v, table, q, k), s["dy"].double(), allow_unused=True)
        out["dtable"] = (torch.zeros_like(table) if dtable is None else dtable).view(case["buckets"], H, 1, 1)
        out = {name: out[name] for name in ("y", "dv", "dtable", "dq", "dk")}
    return out


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------

def work(case):
    """Every input read once, every result written once; the products of the attention and of its gradients (two forward, dP, dV,
    dQ and dK backward) over all keys there can be that a query sees."""
    n = float(case["n"])
    if case["op"] == "layer_norm":
        x = n * case["c"] * case["T"]
        return {"bytes": 4 * ((4 if case["backward"] else 2) * x + 4 * case["c"]), "flops": x * (18 if case["backward"] else 8)}
    if case["op"] == "dropout":
        x = n * case["c"] * case["T"]
        tensors = 2 + case["residual"] + 2 * case["backward"]
        return {"bytes": 4 * tensors * x, "flops": x * (20 + 2 * tensors)}
    Tq, Tk, d = case["Tq"], case["Tk"], case["d"]
    pairs, seen = float(Tq) * Tk, Tk
    if not case["both"]:
        first = 0 if case["at"] == "first" else Tk - Tq
        pairs, seen = float(sum(min(Tk, max(0, i + first + 1)) for i in range(Tq))), min(Tk, Tq + first)
    queries, states = n * case["heads"] * d * Tq, n * case["kv_heads"] * d * seen
    values = (2 * queries + 2 * states) * (2 if case["backward"] else 1)
    product = 2.0 * n * case["heads"] * d * pairs
    return {"bytes": 4 * (values + case["buckets"] * case["heads"]), "flops": product * (6 if case["backward"] else 2)}
