"""How far an attention and its gradients computed in fp32 may be off, vector by vector, from the roundings of their formulas.

u = 2^-24, half a step of fp32. Roundings are taken as independent: a sum of n terms t is off by about u sqrt(n) times the root of the
sum of their squares (the partial sums' roundings), its terms by their own relative errors. With, for a query i and a key j,
  s_ij   score; off by u (sqrt(d) scale sqrt(sum_c (q k)^2) + 3 max_j |s_ij log2 e|) (the product's sum, the multiplication with the scale, the
         reference score that is taken off), and by as much, relative, the weight p_ij
  dp_ij  <dy_i, v_j>: off by u sqrt(d) D_ij, D_ij = sqrt(sum_c (dy v)^2);  <dy_i, y_i> by u sqrt(d) E_i, E_i = sqrt(sum_c (dy y)^2)
the terms of the results, each off by u g_ij, g_ij = sqrt(d) scale sqrt(sum_c (q k)^2) + 5 max_j |s_ij| + sqrt(d) + sqrt(n) + 16, are
  y_i    p_ij v_j                                  n = keys
  dq_i   scale p_ij k_j times dp_ij - dot_i, D_ij   n = keys; and, common to all keys, scale E_i sum_j p_ij k_j
  dk_j   scale p_ij q_i times dp_ij - dot_i, D_ij, E_i     n = queries that read the key
  dv_j   p_ij dy_i                                 n = queries that read the key
and every result is off by u times itself. The 16 is for a handful of roundings: of products (three products of two fp16 parts leave out
2^-24 of one, each part is off by 2^-24), of exp2, of one over the sum. `rss` is the root of the sum of the squares of all that; a vector
(the channels of a query or key) has to be within MARGIN u times the 2-norm of its rss.
"""
import numpy as np

from oracle import ops

U = 2.0 ** -24
MARGIN = 4.0                    # what follows a sum doubles an error once or twice, and a vector is a sample


def split(t, heads):
    t = np.asarray(t, np.float64)
    return t.reshape(t.shape[0], heads, t.shape[1] // heads, -1)


def reference_and_rss(q, k, v, dy, ln, heads, kv_heads, scale):
    """({name: [n][heads][d][tokens]} in 64 bits, the same of rss), for y and, with dy, for dq, dk, dv."""
    scale = float(np.float32(scale))
    p = ops.attention_weights(q, np.where(np.isfinite(k), k, 0), heads, kv_heads, scale, ln)
    n, group, d = p.shape[0], heads // kv_heads, np.shape(q)[1] // heads
    qh, gh = split(q, heads), split(dy, heads) if dy is not None else None
    kh, vh = (ops.counted_values(t, kv_heads, ln) for t in (k, v))
    ref, rss = {}, {}
    for name, like in (("y", qh), ("dq", qh), ("dk", kh), ("dv", kh)):
        if name == "y" or dy is not None:
            ref[name], rss[name] = np.zeros_like(like), np.zeros_like(like)
    for b in range(n):
        for h in range(heads):
            j = h // group
            P, Q, K, V = p[b, h], qh[b, h], kh[b, j], vh[b, j]
            if not P.any():
                continue
            counts = P.any(axis=0)
            s = scale * (Q.T @ K) * counts
            common = np.sqrt(d) * abs(scale) * np.sqrt((Q * Q).T @ (K * K)) + 5 * np.abs(s).max(axis=1, keepdims=True) + np.sqrt(d) + 16
            g = common + np.sqrt(counts.sum())
            y = V @ P.T
            ref["y"][b, h] = y
            rss["y"][b, h] = np.sqrt((V * V) @ (P * P * g * g).T + y * y)
            if dy is None:
                continue
            G = gh[b, h]
            dp = G.T @ V
            dot = (P * dp).sum(axis=1, keepdims=True)
            dS = P * (dp - dot)
            D2, E2 = (G * G).T @ (V * V), (G * G * y * y).sum(axis=0)[:, None]
            ref["dq"][b, h] = scale * (K @ dS.T)
            t2 = (P * g) ** 2 * ((dp - dot) ** 2 + D2)
            shared = scale * (K @ P.T) * np.sqrt(d * E2[:, 0])
            rss["dq"][b, h] = np.sqrt(scale * scale * ((K * K) @ t2.T) + shared ** 2 + ref["dq"][b, h] ** 2)
            g = common + np.sqrt(group * Q.shape[1])
            ref["dk"][b, j] += scale * (Q @ dS)
            rss["dk"][b, j] += scale * scale * ((Q * Q) @ ((P * g) ** 2 * ((dp - dot) ** 2 + D2 + E2)))
            ref["dv"][b, j] += G @ P
            rss["dv"][b, j] += (G * G) @ (P * g) ** 2
    if dy is not None:
        for name in ("dk", "dv"):
            rss[name] = np.sqrt(rss[name] + ref[name] ** 2)
    return ref, rss


def excess(got, ref, rss, axis=2):
    """{name: the largest |error| of a vector over what it may be}; NaN counts as infinitely far off. axis 3: vectors are not the channels
    of a token but a channel's values at all tokens."""
    worst = {}
    for name in ref:
        t = np.asarray(got[name], np.float64).reshape(ref[name].shape)
        off, may = np.sqrt(((t - ref[name]) ** 2).sum(axis=axis)), MARGIN * U * np.sqrt((rss[name] ** 2).sum(axis=axis))
        worst[name] = float(np.max(np.where(np.isfinite(off), off / np.maximum(may, 1e-300), np.inf)))
    return worst


def check(got, q, k, v, dy, ln, heads, kv_heads, scale, what):
    ref, rss = reference_and_rss(q, k, v, dy, ln, heads, kv_heads, scale)
    for axis in (2, 3):
        worst = excess(got, ref, rss, axis)
        assert all(w <= 1.0 for w in worst.values()), (what, axis, worst)
