"""The vocabulary loss where single logits are infinite: what the formula makes of them, in whichever tile, half tile or block of columns they lie.

A row's logits are those of its first channel alone, z = x[:, 0] w[:, 0], with x[:, 0] a power of two and zeros (times finite weights) in the
other channels: exact in fp32, so that -inf and +inf in w[:, 0] make logits of -inf and +inf and nothing else of the row becomes NaN."""
import numpy as np
import pytest
import torch

import paper_2407_12077_b200 as gf

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
INF = float("inf")
# one and several rows through single CTAs (tiles of 128 columns, 64 to a half), and pairs of CTAs (256, two blocks of 64 to a half)
SHAPES = [(1, 700), (5, 700), (130, 1000), (2048, 8192)]


def make(rows, V, z, target, seed=1):
    """x, w, targets with logits z[v] * scale[row], scale one of 1, 2, 0.5; the other channels of w are random, those of x zero."""
    g = torch.Generator().manual_seed(seed)
    D = 64
    x = torch.zeros(rows, D)
    scale = torch.tensor([1.0, 2.0, 0.5])[torch.arange(rows) % 3]
    x[:, 0] = scale
    w = torch.randn(V, D, generator=g)
    w[:, 0] = z
    t = torch.full((rows,), target, dtype=torch.int64)
    return x.to(BF).to(DEV), w.to(BF).to(DEV), t.to(DEV), scale.double().numpy()[:, None] * z.to(BF).double().numpy()[None, :]


def exact(z, target):
    """(loss, lse) in float64; a NaN logit makes both NaN."""
    top = z.max(1)
    with np.errstate(all="ignore"):
        ref = np.where(np.isfinite(top), top, 0.0)
        lse = np.where(np.isinf(top), top, ref + np.log(np.exp(z - ref[:, None]).sum(1)))
        return lse - z[:, target], lse


def same(got, want, want_lse, V, what):
    """Equal where infinite or NaN.  Otherwise: the logits are exact, exponentials off by 2^-20 of themselves, the largest partial sums by a step for each
    addition (64 in a block, one per block of 128 columns), and lse, the logit taken from it and the loss are rounded."""
    got = got.cpu().double().numpy()
    fin = np.isfinite(want)
    assert (np.isnan(got) == np.isnan(want)).all(), what
    assert (got[np.isinf(want)] == want[np.isinf(want)]).all(), what
    bound = 2.0 ** -20 + (64 + V / 128) * 2.0 ** -23 + 2.0 ** -22 * (np.abs(want[fin]) + np.abs(want_lse[fin]))
    assert (np.abs(got[fin] - want[fin]) <= bound).all(), (what, got[fin][:4], want[fin][:4])


def patterns(V):
    def base(v):
        return torch.full((V,), v)

    def put(z, at, v):
        z[at] = v
        return z

    ramp = torch.linspace(-240, -200, V)
    return {
        "a block of 64 masked, the rest far below zero": put(base(-200.0), slice(0, 64), -INF),
        "all but the last columns masked": put(base(-INF), slice(V - 3, V), -300.0),
        "all but one column in the middle masked": put(base(-INF), slice(V // 2, V // 2 + 1), -150.0),
        "every other block masked": put(ramp.clone(), (torch.arange(V) // 64) % 2 == 0, -INF),
        "every other column masked": put(ramp.clone(), torch.arange(V) % 2 == 0, -INF),
        "everything masked": base(-INF),
        "+inf first, large ones behind": put(base(200.0), slice(3, 4), INF),
        "+inf in a later tile": put(base(200.0), slice(V - 5, V - 4), INF),
        "+inf in the middle, masked around it": put(base(-INF), slice(V // 2, V // 2 + 1), INF),
        "+inf twice, in two tiles": put(put(base(-200.0), slice(1, 2), INF), slice(V - 2, V - 1), INF),
        "both infinities": put(put(base(150.0), slice(0, 128), -INF), slice(200, 201), INF),
        "a NaN among masked ones": put(base(-INF), slice(V // 3, V // 3 + 1), float("nan")),
    }


@pytest.mark.parametrize("rows,V", SHAPES)
@pytest.mark.parametrize("which", list(patterns(700)))
def test_loss_and_normaliser(rows, V, which):
    z = patterns(V)[which]
    for target in (V - 2, 2, 200):                   # behind, masked or infinite, depending on the pattern
        x, w, t, logits = make(rows, V, z, target)
        loss, lse = gf.vocab_loss(x, w, t)
        gf.last_device_status()
        if "NaN" in which:
            assert torch.isnan(lse).all() and torch.isnan(loss).all()
            continue
        want, want_lse = exact(logits, target)
        same(lse, want_lse, want_lse, V, which + " lse")
        same(loss, want, want_lse, V, which + " loss")


@pytest.mark.parametrize("rows,V", SHAPES)
@pytest.mark.parametrize("which", ["a block of 64 masked, the rest far below zero", "all but the last columns masked", "every other block masked"])
def test_gradient_under_masked_entries(rows, V, which):
    """dw = P^T x with P exactly zero in masked columns (a masked target's is -1).  P is rounded (2^-8), the result is (2^-8); P's exponential is off by lse's error
    (2^-20 + 128 * 2^-23 + 2^-22 * 480), its argument's rounding (480 * 2^-24), the sum over the rows by (2048 / 16 + 16) 2^-23: under 2^-12 in all."""
    z = patterns(V)[which]
    target = V - 2
    x, w, t, logits = make(rows, V, z, target)
    lse = gf.vocab_loss(x, w, t)[1]
    d = torch.full((rows,), 1.0 / rows, device=DEV)
    dx, dw = gf.vocab_loss_backward(x, w, t, lse, d)
    gf.last_device_status()
    p = np.exp(logits - exact(logits, target)[1][:, None])
    hot = np.zeros_like(p)
    hot[:, target] = 1
    X = x.double().cpu().numpy()
    want, size = ((p - hot) / rows).T @ X, ((p + hot) / rows).T @ X
    got = dw.double().cpu().numpy()
    masked = np.isneginf(z.numpy())
    masked[target] = False
    assert not got[masked].any()
    assert (np.abs(got - want) <= (2 * 2.0 ** -8 + 2.0 ** -12) * size + 2.0 ** -126).all()
    # the masked channel of w meets a P of zero (0 * inf); the others are finite
    assert torch.isfinite(dx[:, 1:]).all()
