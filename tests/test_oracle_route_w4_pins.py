"""Pins for the oracle's router and 4-bit weights: closed forms, differences, and the format's own table."""
import math

import numpy as np
import pytest

import oracle
from oracle import route as orc
from oracle import w4


def test_even_router_has_loss_one_and_no_gradient():
    """Logits that differ by token in which branch leads, evenly: f_b = P_b = 1 / B, so A sum f_b P_b = 1."""
    B = 4
    x = np.zeros((8, B))
    for t in range(8):
        x[t, t % B] = 1.0
    route, p, counts, loss = orc.route_topk(x, 1)
    assert np.array_equal(counts, [2, 2, 2, 2, 8]) and abs(loss - 1.0) < 1e-14
    assert np.allclose(p.sum(1), 1)
    assert np.max(np.abs(orc.route_backward(p, counts, None, 1.0))) < 1e-16


def test_one_branch_for_all_has_loss_near_the_number_of_branches():
    x = np.zeros((5, 6))
    x[:, 2] = 60.0
    route, p, counts, loss = orc.route_topk(x, 1)
    assert np.array_equal(counts, [0, 0, 5, 0, 0, 0, 5]) and abs(loss - 6.0) < 1e-12


def test_ties_bars_padding_and_empty_rows():
    inf = np.inf
    x = np.array([[1., 1, 1, 1], [-inf, 0, -inf, -inf], [-inf] * 4, [0, 1, 2, 3], [np.nan, 0, 1, -1]])
    route, p, counts, loss = orc.route_topk(x, 2, active=[1, 1, 0, 1], real=[1, 1, 1, 0, 1])
    assert route.tolist() == [[1, 1, 0, 0], [0, 1, 0, 0], [0] * 4, [0] * 4, [0, 1, 0, 1]]
    assert counts.tolist() == [1, 3, 0, 1, 3]
    assert np.allclose(p[0], [1 / 3, 1 / 3, 0, 1 / 3]) and np.array_equal(p[1], [0, 1, 0, 0]) and not p[2:4].any()
    assert np.isnan(p[4, [0, 1, 3]]).all() and p[4, 2] == 0 and np.isnan(loss)


@pytest.mark.parametrize("dloss", [0.0, 0.7])
def test_gradient_against_differences(dloss):
    """The counts are steps of the logits: with them held, the loss is a smooth function whose differences are the gradient."""
    rng = np.random.default_rng(3)
    T, B, k = 7, 5, 2
    x = rng.standard_normal((T, B))
    x[2, 1] = -np.inf
    active = np.array([1, 1, 1, 0, 1])
    real = np.array([1, 1, 1, 1, 0, 1, 1])
    dp = rng.standard_normal((T, B))
    _, p, counts, _ = orc.route_topk(x, k, active, real)

    def value(y):
        _, q, _, _ = orc.route_topk(y, k, active, real)
        f = counts[:B] / counts[:B].sum()
        return float(np.sum(dp * q)) + dloss * 4 * float(np.sum(f * q.sum(0))) / counts[B]

    d = orc.route_backward(p, counts, dp, dloss, n_active=4)
    eps = 1e-6
    for t in range(T):
        for b in range(B):
            if not np.isfinite(x[t, b]):
                assert d[t, b] == 0
                continue
            up, down = x.copy(), x.copy()
            up[t, b] += eps
            down[t, b] -= eps
            assert abs((value(up) - value(down)) / (2 * eps) - d[t, b]) < 1e-8, (t, b)


def test_every_code_keeps_its_value():
    """A block that holds 6 and all sixteen elements times a power of two is kept as it is."""
    row = np.array([m * s for m in w4.MAGNITUDES for s in (1.0, -1.0)] * 2)
    for e in (-120, -3, 0, 5, 100):
        W = np.ldexp(row, e)[None, :]
        codes, scales = w4.quantize(W)
        assert scales[0, 0] == 127 + e
        assert np.array_equal(w4.dequantize(codes, scales), W)
        assert np.array_equal(np.signbit(w4.dequantize(codes, scales)), np.signbit(W))


def test_halfway_and_saturation():
    for a, want in ((0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5.0, 4), (7.9, 6), (0.26, 0.5), (5.01, 6)):
        assert w4.MAGNITUDES[w4.nearest_code(a)] == want, a
    W = np.zeros((1, 32))
    W[0, 0], W[0, 1] = 7.75, 1.25            # the largest has the exponent of 4: scale 1
    codes, scales = w4.quantize(W)
    assert scales[0, 0] == 127 and w4.dequantize(codes, scales)[0, :2].tolist() == [6.0, 1.0]


def test_error_is_at_most_half_a_step():
    rng = np.random.default_rng(0)
    W = rng.standard_normal((4, 96)) * 0.02
    v = w4.dequantize(*w4.quantize(W))
    top = np.repeat(np.abs(W.reshape(4, 3, 32)).max(2), 32, axis=1)
    unit = np.exp2(np.floor(np.log2(top)) - 2)
    # steps of half a unit below 2 units, of a unit to 4, of 2 to 8, whose upper half is cut at 6
    assert np.all(np.abs(v - W) <= np.where(np.abs(W) > 6 * unit, 2 * unit, np.maximum(unit / 4, np.abs(W) / 5 + 1e-15)))


def test_blocks_that_are_not_finite_and_zero():
    W = np.zeros((2, 64))
    W[0, 3] = math.inf
    W[1, 40] = math.nan
    codes, scales = w4.quantize(W)
    assert scales.tolist() == [[255, 1], [1, 255]] and not codes.any()
    v = w4.dequantize(codes, scales)
    assert np.isnan(v[0, :32]).all() and not v[0, 32:].any() and np.isnan(v[1, 32:]).all()


def test_forward_of_dequantised_weights_is_linear_in_the_scales_of_down():
    """One exponent more on all of W_down doubles the result."""
    rng = np.random.default_rng(1)
    Wg, Wu = (w4.dequantize(*w4.quantize(rng.standard_normal((64, 32)) * 0.1)) for _ in range(2))
    codes, scales = w4.quantize(rng.standard_normal((32, 64)) * 0.1)
    x = rng.standard_normal((3, 32)).astype(np.float32)
    off, alpha, mask = np.array([0, 20, 64], np.int32), np.array([1.0, 0.5], np.float32), np.ones(2, np.uint8)
    f = [oracle.mlpmoe_forward(x, Wg.astype(np.float32), Wu.astype(np.float32), w4.dequantize(codes, scales + d).astype(np.float32),
                               off, alpha, mask) for d in (0, 1)]
    assert np.allclose(2 * np.asarray(f[0], np.float64), f[1], rtol=1e-6)
