"""Pins of the oracle's operators around the recurrence (gradient of the norm, gated linear block, vocabulary loss) to facts that do
not come from the oracle: brute-force loops, closed forms, central differences."""
import math

import numpy as np
import pytest

from oracle import wkv6_oracle as orc

H = 1e-6


def difference(f, a):
    """Gradient of the scalar f() with respect to the array a by central differences (a is put back)."""
    g = np.zeros_like(a)
    for i in np.ndindex(a.shape):
        keep = a[i]
        a[i] = keep + H
        up = f()
        a[i] = keep - H
        g[i] = (up - f()) / (2 * H)
        a[i] = keep
    return g


# central differences: the third derivative times H^2 and 1e-16 / H of cancellation, both below 1e-9 at these magnitudes
CLOSE = dict(rtol=1e-7, atol=2e-8)


@pytest.mark.parametrize("affine", [False, True])
def test_norm_gradient_is_that_of_the_norm(affine):
    rng = np.random.default_rng(1)
    y, dout = rng.normal(size=(2, 3, 2, 4)), rng.normal(size=(2, 3, 2, 4))
    gamma, beta = (rng.normal(size=8), rng.normal(size=8)) if affine else (np.ones(8), np.zeros(8))
    f = lambda: float((orc.layernorm_heads(y, gamma, beta, 1e-3) * dout).sum())  # noqa: E731
    dy, dg, db = orc.layernorm_heads_backward(y, dout, gamma if affine else None, 1e-3)
    np.testing.assert_allclose(dy, difference(f, y), **CLOSE)
    np.testing.assert_allclose(dg, difference(f, gamma), **CLOSE)
    np.testing.assert_allclose(db, difference(f, beta), **CLOSE)


@pytest.mark.parametrize("act,at", [("sigmoid", [(0.0, 0.5), (math.log(3), 0.75)]), ("relu2", [(-2.0, 0.0), (0.0, 0.0), (3.0, 9.0)]),
                                    ("silu", [(0.0, 0.0), (math.log(3), 0.75 * math.log(3))]), ("gelu", [(0.0, 0.0), (1.0, 0.8413447460685429)])])
def test_activations_at_known_points(act, at):
    for a, v in at:
        assert abs(orc.activation(np.array([a]), act)[0][0] - v) < 1e-15


@pytest.mark.parametrize("act", ["sigmoid", "relu2", "silu", "gelu"])
@pytest.mark.parametrize("second", ["none", "same", "own"])
def test_gated_linear_by_loops_and_its_gradient_by_differences(act, second):
    rng = np.random.default_rng(2)
    x, w, dy = rng.normal(size=(3, 4)), rng.normal(size=(4, 5)), rng.normal(size=(3, 5))
    x2 = rng.normal(size=(3, 2)) if second == "own" else None
    w2 = None if second == "none" else rng.normal(size=(4 if second == "same" else 2, 5))
    y = orc.gated_linear(x, w, x2, w2, act)
    v = x if x2 is None else x2
    for i in range(3):
        for j in range(5):
            a = sum(x[i, k] * w[k, j] for k in range(4))
            f = {"sigmoid": 1 / (1 + math.exp(-a)), "relu2": max(a, 0) ** 2, "silu": a / (1 + math.exp(-a)),
                 "gelu": a * 0.5 * (1 + math.erf(a / math.sqrt(2)))}[act]
            b = 1.0 if w2 is None else sum(v[i, k] * w2[k, j] for k in range(v.shape[1]))
            assert abs(y[i, j] - f * b) < 1e-13
    got = orc.gated_linear_backward(x, w, dy, x2, w2, act)
    f = lambda: float((orc.gated_linear(x, w, x2, w2, act) * dy).sum())  # noqa: E731
    for g, a in zip(got, (x, w, x2, w2)):
        assert (g is None) == (a is None)
        if a is not None:
            np.testing.assert_allclose(g, difference(f, a), **CLOSE)


def test_loss_of_equal_logits_is_the_logarithm_of_the_vocabulary():
    loss, lse = orc.vocab_loss(np.ones((3, 4)), np.full((7, 4), 0.25), np.array([0, 6, -100]))
    np.testing.assert_allclose(lse, 1 + math.log(7), rtol=1e-14)
    np.testing.assert_allclose(loss, [math.log(7), math.log(7), 0.0], rtol=1e-14)


def test_loss_by_loops_and_its_gradient_by_differences():
    rng = np.random.default_rng(3)
    x, w, d = rng.normal(size=(4, 3)), rng.normal(size=(6, 3)), rng.normal(size=4)
    t = np.array([5, -1, 0, 6])
    loss, lse = orc.vocab_loss(x, w, t)
    for i in range(4):
        z = [sum(x[i, k] * w[v, k] for k in range(3)) for v in range(6)]
        s = math.log(sum(math.exp(q) for q in z))
        assert abs(lse[i] - s) < 1e-13
        assert abs(loss[i] - (s - z[t[i]] if 0 <= t[i] < 6 else 0.0)) < 1e-13
    f = lambda: float((orc.vocab_loss(x, w, t)[0] * d).sum())  # noqa: E731
    dx, dw, P = orc.vocab_loss_backward(x, w, t, d)
    np.testing.assert_allclose(dx, difference(f, x), **CLOSE)
    np.testing.assert_allclose(dw, difference(f, w), **CLOSE)
    assert not P[1].any() and not P[3].any()
    np.testing.assert_allclose(P.sum(1), 0, atol=1e-15)
