"""Pins of the oracle's layer norm, dropout, position bias and biased attention: torch in 64 bits, central differences, published vectors
of the generator, and buckets written down by hand."""
import numpy as np
import pytest
import torch

import workloads
from oracle import ops
from oracle.backward import attention_vjp, backward, layer_norm_vjp, position_bias_vjp
from oracle.forward import forward


@pytest.fixture(autouse=True)
def fp64_storage(monkeypatch):
    monkeypatch.setattr(ops, "_out", lambda x: np.ascontiguousarray(x, dtype=np.float64))


@pytest.mark.parametrize("shape", [(2, 7, 2, 3), (1, 1, 1, 1), (3, 2, 1, 5)])
def test_layer_norm_and_its_gradients(shape):
    rng = np.random.default_rng(3)
    x, dy = rng.standard_normal((2,) + shape)
    gamma, beta = rng.standard_normal((2, shape[1]))
    xt, gt, bt = (torch.tensor(t, requires_grad=True) for t in (x, gamma, beta))
    y = torch.nn.functional.layer_norm(xt.permute(0, 2, 3, 1), (shape[1],), gt, bt, 1e-3).permute(0, 3, 1, 2)
    np.testing.assert_allclose(ops.layer_norm(x, gamma, beta, 1e-3), y.detach().numpy(), rtol=0, atol=1e-12)
    for got, ref in zip(layer_norm_vjp(x, gamma, 1e-3, dy), torch.autograd.grad(y, (xt, gt, bt), torch.tensor(dy))):
        np.testing.assert_allclose(got, ref.numpy(), rtol=0, atol=1e-11)


def test_generator_gives_its_published_vectors():
    """Known answers of Philox4x32-10 that its authors publish with it."""
    ones = 0xFFFFFFFF
    pi = (0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344)
    for counter, key, words in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                                ((ones,) * 4, (ones,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                                (pi, (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(ops.philox4x32(np.array([counter], np.uint32), key)[0]) == words


def test_dropout_keeps_its_share_and_drops_what_is_not_finite():
    seed = np.array([12345.0, 1.0], np.float32).reshape(1, 1, 1, 2)
    for rate in (0.0, 0.1, 0.5, 0.9):
        m = ops.dropout_scale((3, 50, 7, 13), seed, rate, 2)
        n, kept = m.size, int((m > 0).sum())
        assert abs(kept - n * (1 - rate)) <= 5 * np.sqrt(n * rate * (1 - rate)), rate
        # the rate as fp32, then rounded to 2^-32, at most half of that off
        assert set(np.unique(m)) <= {0.0, m.max()} and abs(m.max() * (1 - float(np.float32(rate))) - 1) <= 2.0 ** -32 / (1 - rate)
    a, b, c = (ops.dropout_scale((1, 4, 9, 9), seed + d, 0.5, site) for d, site in ((0, 0), (0, 1), (1, 0)))
    assert (a != b).any() and (a != c).any() and (b != c).any()
    x = np.full((1, 1, 1, 64), np.nan)
    y = ops.dropout(x, seed, None, 0.5, 0)
    assert np.isnan(y).sum() == (ops.dropout_scale(x.shape, seed, 0.5, 0) > 0).sum() < 64


def test_position_buckets_by_hand():
    def of(far, *how):
        return [ops.position_bucket(d, *how) for d in far]

    # 32 buckets, both directions, 128: 8 exact ones, then steps of a factor sqrt 2, each border exactly on a whole number or between two
    assert of(range(0, -9, -1), 32, 128, True) == [0, 1, 2, 3, 4, 5, 6, 7, 8]
    assert of([-11, -12, -15, -16, -22, -23, -31, -32, -45, -46, -63, -64, -90, -91, -127, -128, -5000], 32, 128, True) == \
        [8, 9, 9, 10, 10, 11, 11, 12, 12, 13, 13, 14, 14, 15, 15, 15, 15]
    assert of([1, 7, 8, 128, 1000], 32, 128, True) == [17, 23, 24, 31, 31]
    assert of([0, -1, -15, -16, -17, -128, -129, 1, 99], 32, 128, False) == [0, 1, 15, 16, 16, 31, 31, None, None]
    assert of([-1, 0, 1, -2, 2], 4, 2, True) == [1, 0, 3, 1, 3]


def test_position_bias_and_its_gradient():
    rng = np.random.default_rng(5)
    for buckets, m, both in ((8, 10, True), (5, 9, False), (32, 128, True)):
        table, dbias = rng.standard_normal((buckets, 3)), rng.standard_normal((1, 3, 1, 2 * m + 1))
        bias = ops.position_bias(table, 3, buckets, m, both)
        assert bias.shape == dbias.shape and np.isneginf(bias).sum() == (0 if both else 3 * m)
        dtable = position_bias_vjp(dbias, 3, buckets, m, both)
        step = rng.standard_normal(table.shape)
        moved = ops.position_bias(table + step, 3, buckets, m, both)
        seen = np.isfinite(bias)
        np.testing.assert_allclose(((moved[seen] - bias[seen]) * dbias[seen]).sum(), (step * dtable).sum(), atol=1e-12)


@pytest.mark.parametrize("at", ["first", "last"])
@pytest.mark.parametrize("lengths", [None, [9, 4, 0]])
def test_biased_attention_and_its_gradients(at, lengths):
    rng = np.random.default_rng(7)
    n, heads, kv, d, tq, tk, m = 3, 4, 2, 3, 6, 9, 4
    q, dy = rng.standard_normal((2, n, heads * d, 1, tq))
    k, v = rng.standard_normal((2, n, kv * d, 1, tk))
    bias = rng.standard_normal((1, heads, 1, 2 * m + 1))
    bias[0, 1, 0, m + 1:] = -np.inf                              # this head only looks back: with "last" and few keys some queries see none
    ln = None if lengths is None else np.array(lengths, np.float32).reshape(n, 1, 1, 1)
    leaves = [torch.tensor(t, requires_grad=True) for t in (q, k, v, np.where(np.isfinite(bias), bias, 0.0))]
    qt, kt, vt, bt = leaves
    out = []
    for b in range(n):
        keys = tk if lengths is None else lengths[b]
        for h in range(heads):
            ys = []
            for i in range(tq):
                offset = keys - tq if at == "last" else 0
                away = [min(max(j - i - offset, -m), m) + m for j in range(keys)]
                seen = [j for j in range(keys) if np.isfinite(bias[0, h, 0, away[j]])]
                if not seen:
                    ys.append(torch.zeros(d, dtype=torch.float64))
                    continue
                j = h // (heads // kv)
                score = torch.stack([0.4 * (qt[b, h * d:(h + 1) * d, 0, i] * kt[b, j * d:(j + 1) * d, 0, t]).sum() + bt[0, h, 0, away[t]] for t in seen])
                ys.append((torch.softmax(score, 0)[None] * vt[b, j * d:(j + 1) * d, 0, seen]).sum(1))
            out.append(torch.stack(ys, 1))
    y = torch.stack(out).reshape(n, heads * d, 1, tq)
    np.testing.assert_allclose(ops.attention(q, k, v, ln, heads, kv, 0.4, bias, at), y.detach().numpy(), rtol=0, atol=1e-12)
    for got, ref in zip(attention_vjp(q, k, v, ln, heads, kv, 0.4, dy, bias, at), torch.autograd.grad(y, leaves, torch.tensor(dy))):
        np.testing.assert_allclose(got, ref.numpy(), rtol=0, atol=1e-11)


@pytest.mark.parametrize("both", [True, False])
def test_gradients_of_a_block_by_differences(both):
    w = workloads.transformer_block(both=both)
    rng = np.random.default_rng(2)
    out = w.outputs[0]
    seed = rng.standard_normal(w.nodes[out].shape)
    _, d_weight = backward(w, {out: seed})
    for v, nd in enumerate(w.nodes):
        for j, keep in enumerate(nd.weights):
            step = rng.standard_normal(keep.shape)
            side = []
            for h in (1e-5, -1e-5):
                nd.weights[j] = keep.astype(np.float64) + h * step
                side.append((forward(w)[out].astype(np.float64) * seed).sum())
            nd.weights[j] = keep
            found, stated = (side[0] - side[1]) / 2e-5, (step * d_weight[v][j]).sum()
            # the function's curvature over 1e-5, and values near 0 whose ReLU changes side
            assert abs(found - stated) <= 1e-5 * max(1.0, np.abs(step * d_weight[v][j]).sum()), (v, nd.op, j, found, stated)
