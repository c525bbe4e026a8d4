"""The operators around the recurrence on the GPU (gradient of the norm, gated linear block and its gradient, vocabulary loss and its
gradient) against the float64 oracle, element by element.

Bounds are sums of the roundings on an element's way.  HALF = 2^-8 is half a step of bf16 relative to the value: one for a result,
one for an operand that a kernel rounds on the way (da, db, P), carried through the product as HALF * |operand| |other factor|.  A
product over K indices is summed in fp32 in runs of 16: K/16 + 16 additions, each off by at most one step (2^-23) of a partial sum,
which is at most the sum of the magnitudes.  The activations' exponential is off by 2 + 1.2 |a| steps and the division by 2: with
|a| < 60, under 2^-16 of the value."""
import numpy as np
import pytest
import torch

import paper_2407_12077_b200 as gf
from oracle import wkv6_oracle as orc

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -8
BF = torch.bfloat16
CANARY = 777.0


def acc(k):
    return (k / 16 + 16) * 2.0 ** -23


def normal(g, *shape, std=1.0, dtype=BF):
    return (torch.randn(*shape, generator=g) * std).to(dtype)


def np64(t):
    return t.detach().cpu().double().numpy()


def near(got, want, bound, what):
    got = np64(got)
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.nanmax(np.abs(got - want) / np.broadcast_to(bound, got.shape)):.2f} of the bound"


def dev(*ts):
    return [None if t is None else t.to(DEV) for t in ts]


# ------------------------------------------------------------------------------------------------ gradient of the norm
# every (slices per lane, warps per row) variant of either type, full and ragged
WIDTHS = [(1, 8), (1, 64), (4, 64), (5, 64), (8, 64), (12, 64), (16, 64), (20, 64), (31, 64), (32, 64), (33, 64), (40, 64), (64, 64), (65, 64),
          (96, 64), (100, 64), (128, 64), (7, 24), (45, 8)]


def norm_bounds(y, dout, gamma, eps, dtype):
    """Bounds of (dy, dgamma, dbeta): every term in fp32 is off by some 40 steps of its own magnitude (sums over lanes and warps, the
    reciprocal square root), sums over rows by one step each of the sum of magnitudes."""
    y, dout = (np64(t).reshape(len(t), -1) for t in (y, dout))
    D = y.shape[1]
    gm = np.ones(D) if gamma is None else np64(gamma).reshape(D)
    mu = y.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((y - mu) ** 2).mean(1, keepdims=True) + eps)
    # the mean is off by steps of the largest magnitude, and with it every deviation
    dev_ = np.abs(y - mu) + 8 * np.abs(y).max(1, keepdims=True)
    xh = dev_ * rstd
    g = np.abs(dout * gm)
    terms = rstd * (g + g.mean(1, keepdims=True) + xh * (g * xh).mean(1, keepdims=True))
    u = 40 * 2.0 ** -23
    dy = u * terms
    rows = len(y)
    return dy, (u + rows * 2.0 ** -23) * (np.abs(dout) * xh).sum(0), (rows * 2.0 ** -23) * np.abs(dout).sum(0)


def check_norm(y, dout, gamma, eps, got, what):
    want = orc.layernorm_heads_backward(y, dout, gamma, eps)
    bounds = norm_bounds(y, dout, gamma, eps, y.dtype)
    first = bounds[0].reshape(want[0].shape) + (HALF if y.dtype == BF else 2.0 ** -24) * np.abs(want[0])
    near(got[0], want[0], first, what + " dy")
    for n, a, b, c in zip(("dgamma", "dbeta"), got[1:], want[1:], bounds[1:]):
        near(a, b, c + 2.0 ** -24 * np.abs(b), f"{what} {n}")


@pytest.mark.parametrize("rows", [1, 3, 9, 1001])
@pytest.mark.parametrize("H,N", WIDTHS)
@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_norm_gradient_over_widths(rows, H, N, dtype):
    g = torch.Generator().manual_seed(rows + H * N)
    y, dout, gamma = normal(g, rows, H, N, std=2, dtype=dtype) + 0.3, normal(g, rows, H, N, dtype=dtype), 1 + normal(g, H * N, std=0.5, dtype=torch.float32)
    yd, dd, gd = dev(y, dout, gamma)
    room = torch.full((rows + 2, H, N), CANARY, dtype=dtype, device=DEV)
    got = gf.layernorm_heads_backward(yd, dd, gd, 1e-5, dy=room[1:rows + 1])
    gf.last_device_status()
    assert torch.all(room[0] == CANARY) and torch.all(room[-1] == CANARY)
    check_norm(y, dout, gamma, 1e-5, got, f"rows {rows} D {H * N}")


@pytest.mark.parametrize("dtype", [BF, torch.float32])
def test_norm_gradient_in_place_without_gamma_and_without_sums(dtype):
    g = torch.Generator().manual_seed(3)
    y, dout = normal(g, 37, 32, 64, dtype=dtype), normal(g, 37, 32, 64, dtype=dtype)
    want = gf.layernorm_heads_backward(*dev(y, dout), None, 0.5)
    check_norm(y, dout, None, 0.5, want, "no gamma")
    yd, dd = dev(y, dout)
    assert torch.equal(gf.layernorm_heads_backward(yd, dd, None, 0.5, dy=dd)[0], want[0])
    dd = dout.to(DEV)
    got = gf.layernorm_heads_backward(yd, dd, None, 0.5, want_params=False, dy=yd)
    assert torch.equal(got[0], want[0]) and got[1] is None and got[2] is None


def test_norm_gradient_with_a_gamma_that_has_to_be_copied():
    g = torch.Generator().manual_seed(8)
    y, dout, wide = dev(normal(g, 50, 4, 64), normal(g, 50, 4, 64), torch.randn(4, 128, generator=g))
    gamma = wide[:, :64]
    want = gf.layernorm_heads_backward(y, dout, gamma.contiguous())
    for _ in range(3):
        got = gf.layernorm_heads_backward(y, dout, gamma)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norm_gradient_of_a_constant_row_and_of_no_rows():
    y, dout = torch.full((2, 4, 64), 3.0, device=DEV), torch.ones(2, 4, 64, device=DEV)
    dy, dg, db = gf.layernorm_heads_backward(y, dout, None, 1e-5)       # deviations and the centred gradient are exactly zero
    assert not dy.any() and not dg.any() and torch.all(db == 2)
    none = torch.empty(0, 4, 64, device=DEV)
    dy, dg, db = gf.layernorm_heads_backward(none, none, None, 1e-5)
    assert dy.shape == (0, 4, 64) and not dg.any() and not db.any()


def test_norm_gradient_keeps_a_nan_to_its_row():
    g = torch.Generator().manual_seed(4)
    y, dout = dev(normal(g, 300, 8, 64), normal(g, 300, 8, 64))
    clean = gf.layernorm_heads_backward(y, dout)[0]
    y[100, 3, 5] = float("nan")
    dy, dg, _ = gf.layernorm_heads_backward(y, dout)
    keep = torch.arange(300, device=DEV) != 100
    assert torch.equal(dy[keep], clean[keep]) and torch.isnan(dy[100]).all() and torch.isnan(dg).all()


# ------------------------------------------------------------------------------------------------ gated linear block
ACTS = ["sigmoid", "relu2", "silu", "gelu"]


def gate_parts(x, w, x2, w2, act):
    """a, b, the activation and its derivative, and bounds on what fp32 makes of them: (a, da, b, db, f, ef, df, edf)."""
    X, W = np64(x), np64(w)
    a, ea = X @ W, acc(W.shape[0]) * (np.abs(X) @ np.abs(W))
    f, df = orc.activation(a, act)
    # second derivatives: sigmoid < 0.1, silu < 0.5, gelu < 0.8, relu^2 2
    ef = (np.abs(df) + 2 * ea) * ea + 2.0 ** -16 * np.abs(f)
    edf = 2 * ea + 2.0 ** -16 * (np.abs(df) + (np.abs(a) < 20) * (1.0 if act in ("silu", "gelu") else 0.0))
    b, eb = np.ones_like(a), np.zeros_like(a)
    if w2 is not None:
        X2, W2 = np64(x if x2 is None else x2), np64(w2)
        b, eb = X2 @ W2, acc(W2.shape[0]) * (np.abs(X2) @ np.abs(W2))
    return a, ea, b, eb, f, ef, df, edf


def make_gate(rows, K1, K2, F, seed):
    """K2 = 0: x2 is x; -1: no second product."""
    g = torch.Generator().manual_seed(seed)
    x, w = normal(g, rows, K1), normal(g, K1, F, std=K1 ** -0.5)
    x2 = normal(g, rows, K2) if K2 > 0 else None
    w2 = normal(g, K2 or K1, F, std=(K2 or K1) ** -0.5) if K2 >= 0 else None
    return x, w, x2, w2, normal(g, rows, F)


def check_gate(x, w, x2, w2, act, out, what):
    a, ea, b, eb, f, ef, df, edf = gate_parts(x, w, x2, w2, act)
    want = f * b
    near(out, want, HALF * np.abs(want) + (ef * (np.abs(b) + eb) + np.abs(f) * eb) * (1 + HALF) + 2.0 ** -126, what)


def check_gate_grad(x, w, x2, w2, act, dy, got, what):
    a, ea, b, eb, f, ef, df, edf = gate_parts(x, w, x2, w2, act)
    d = np.abs(np64(dy))
    want = orc.gated_linear_backward(x, w, dy, x2, w2, act)
    X, W = np64(x), np64(w)
    da, db = np64(dy) * b * df, np64(dy) * f
    eda = HALF * np.abs(da) + (1 + HALF) * d * (edf * (np.abs(b) + eb) + np.abs(df) * eb)
    edb = HALF * np.abs(db) + (1 + HALF) * d * ef
    ada, adb = np.abs(da) + eda, np.abs(db) + edb
    rows, F = d.shape
    V = X if x2 is None else np64(x2)
    ex = eda @ np.abs(W.T) + acc(F) * (ada @ np.abs(W.T))
    ew = np.abs(X.T) @ eda + acc(rows) * (np.abs(X.T) @ ada)
    e2 = e2w = None
    if w2 is not None:
        W2 = np64(w2)
        e2 = edb @ np.abs(W2.T) + acc(F) * (adb @ np.abs(W2.T))
        e2w = np.abs(V.T) @ edb + acc(rows) * (np.abs(V.T) @ adb)
        if x2 is None:
            ex, e2 = ex + e2 + acc(2 * F) * (ada @ np.abs(W.T)), None
    for n, g, t, e in zip(("dx", "dw", "dx2", "dw2"), got, want, (ex, ew, e2, e2w)):
        assert (g is None) == (t is None)
        if t is not None:
            near(g, t, HALF * np.abs(t) + (1 + HALF) * e + 2.0 ** -126, f"{what} {n}")


# one row to several tiles; depths and widths on both sides of 64, 128, 256; single CTAs, clusters, pairs of CTAs (the large ones)
GATES = [(1, 64, -1, 64), (1, 2048, 0, 200), (3, 72, 136, 8), (7, 8, 8, 8), (64, 128, 0, 64), (65, 136, -1, 136), (127, 64, 200, 72), (128, 256, 0, 128),
         (129, 200, 328, 264), (333, 768, 0, 328), (600, 72, -1, 2056), (2500, 136, 200, 4008), (2305, 72, 0, 4104), (1900, 264, 328, 2304), (4096, 64, -1, 2560)]


@pytest.mark.parametrize("rows,K1,K2,F", GATES)
@pytest.mark.parametrize("act", ACTS)
def test_gated_linear_matches_oracle(rows, K1, K2, F, act):
    x, w, x2, w2, _ = make_gate(rows, K1, K2, F, seed=rows + K1)
    room = torch.full((rows + 2, F), CANARY, dtype=BF, device=DEV)
    before = gf.launch_count()
    gf.gated_linear(*dev(x, w, x2, w2), act=act, out=room[1:rows + 1])
    gf.last_device_status()
    assert gf.launch_count() - before == 1
    assert torch.all(room[0] == CANARY) and torch.all(room[-1] == CANARY)
    check_gate(x, w, x2, w2, act, room[1:rows + 1], f"{rows} {K1} {K2} {F} {act}")


@pytest.mark.parametrize("rows,K1,K2,F", [s for s in GATES if s[0] < 4000])
@pytest.mark.parametrize("act", ACTS)
def test_gated_linear_gradient_matches_oracle(rows, K1, K2, F, act):
    x, w, x2, w2, dy = make_gate(rows, K1, K2, F, seed=rows + K1 + 1)
    got = gf.gated_linear_backward(*dev(x, w, dy, x2, w2), act=act)
    gf.last_device_status()
    check_gate_grad(x, w, x2, w2, act, dy, got, f"{rows} {K1} {K2} {F} {act}")


def test_gated_linear_gradient_agrees_with_differences_of_the_forward_call():
    """Directional differences of the forward call itself.  Its outputs are off by HALF of their values each; over the whole tensor,
    weighted with dy of random sign, these add up like a random walk: 6 of its standard deviations."""
    x, w, x2, w2, dy = make_gate(256, 128, 72, 136, seed=9)
    x, w, x2, w2, dy = dev(x, w, x2, w2, dy)
    grads = gf.gated_linear_backward(x, w, dy, x2, w2, act="silu")
    g = torch.Generator(device=DEV).manual_seed(10)
    for t, grad in zip((x, w, x2, w2), grads):
        t0 = t.clone()
        step = 0.25 * t0.float().square().mean().sqrt() * torch.randn(t.shape, generator=g, device=DEV)
        ups, downs = (t0 + step).to(BF), (t0 - step).to(BF)
        taken = (ups.double() - downs.double())
        outs = []
        for v in (ups, downs):
            t.copy_(v)
            outs.append(gf.gated_linear(x, w, x2, w2, act="silu").double())
        t.copy_(t0)
        diff = ((outs[0] - outs[1]) * dy.double()).sum()
        noise = (HALF / 3 ** 0.5) * ((outs[0].square() + outs[1].square()) * dy.double().square()).sum().sqrt()
        along = (grad.double() * taken).sum()
        # the cubic remainder of a central difference over this step stays below 4 % of the gradient's own scale
        scale = grad.double().norm() * taken.norm()
        assert abs(diff - along) <= 6 * noise + 0.04 * scale, (float(diff), float(along))


def test_gated_linear_with_leading_dimensions_and_of_nothing():
    x, w, x2, w2, _ = make_gate(60, 64, 72, 136, seed=5)
    y = gf.gated_linear(*dev(x, w, x2, w2), act="sigmoid")
    y3 = gf.gated_linear(*dev(x.view(3, 4, 5, 64), w, x2.view(3, 4, 5, 72), w2), act="sigmoid")
    assert torch.equal(y3.view(60, 136), y)
    e, e2, dy = (torch.empty(0, n, dtype=BF, device=DEV) for n in (64, 72, 136))
    assert gf.gated_linear(e, w.to(DEV), e2, w2.to(DEV)).shape == (0, 136)
    dx, dw, dx2, dw2 = gf.gated_linear_backward(e, w.to(DEV), dy, e2, w2.to(DEV))
    assert dx.shape == (0, 64) and dx2.shape == (0, 72) and not dw.any() and not dw2.any()


@pytest.mark.parametrize("act", ACTS)
def test_gated_linear_extreme_values(act):
    """Products far outside the exponential's range, zeros, and what a NaN or an infinity in one row leaves of the others."""
    w = torch.eye(64).to(BF)
    x = torch.zeros(8, 64)
    x[0], x[1], x[2, ::2], x[3, ::2] = 200.0, -200.0, 88.0, -88.0
    x[4, 7], x[5, 7], x[6, 7] = float("nan"), float("inf"), float("-inf")
    x = x.to(BF)
    y = np64(gf.gated_linear(x.to(DEV), w.to(DEV), act=act))
    gf.last_device_status()
    want = orc.gated_linear(x[:4], w, act=act)
    assert (np.abs(y[:4] - want) <= HALF * np.abs(want) + 2.0 ** -20).all()
    assert np.isnan(y[4]).all() and np.isnan(y[5]).any() and np.isnan(y[6]).any()       # 0 * inf is among the row's products
    assert np.isfinite(y[7]).all()


# ------------------------------------------------------------------------------------------------ vocabulary loss
LOSSES = [(1, 64, 1), (1, 128, 500), (5, 8, 7), (7, 768, 4001), (63, 72, 129), (128, 136, 1000), (129, 64, 257), (300, 200, 4096), (2500, 64, 20011), (2304, 136, 33000)]


def make_loss(rows, D, V, seed, std=2.0):
    g = torch.Generator().manual_seed(seed)
    x, w = normal(g, rows, D), normal(g, V, D, std=std * D ** -0.5)
    t = torch.randint(0, V, (rows,), generator=g)
    t[::7] = -100
    t[3::50] = V                                     # just past the vocabulary: no target either
    t[1::40] = V - 1
    return x, w, t, torch.randn(rows, generator=g)


def logit_error(x, w):
    """Per row, how far fp32 logits may be off: the largest over the vocabulary."""
    return acc(x.shape[1]) * (np.abs(np64(x)) @ np.abs(np64(w)).T).max(1)


@pytest.mark.parametrize("rows,D,V", LOSSES)
def test_vocab_loss_matches_oracle(rows, D, V):
    x, w, t, _ = make_loss(rows, D, V, seed=rows + V)
    loss, lse = gf.vocab_loss(*dev(x, w, t))
    gf.last_device_status()
    want, want_lse = orc.vocab_loss(x, w, t)
    # exponentials off by 2^-20 of themselves at most, the largest partial sums by a step for each of V/4 additions per tile of 256 and each tile
    e = logit_error(x, w) + 2.0 ** -20 + (64 + V / 128) * 2.0 ** -23
    near(lse, want_lse, e + 2.0 ** -23 * np.abs(want_lse), "lse")
    near(loss, want, 2 * e + 2.0 ** -22 * (np.abs(want_lse) + np.abs(want)), "loss")
    none = (t < 0) | (t >= V)
    assert not loss.cpu()[none].any()


@pytest.mark.parametrize("rows,D,V", LOSSES)
@pytest.mark.parametrize("weighted", [False, True])
def test_vocab_loss_gradient_matches_oracle(rows, D, V, weighted):
    x, w, t, d = make_loss(rows, D, V, seed=rows + V + 1)
    d = d if weighted else None
    xd, wd, td, dd = dev(x, w, t, d)
    lse = gf.vocab_loss(xd, wd, td)[1]
    got = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    dx, dw, P = orc.vocab_loss_backward(x, w, t, d)
    scale = np.ones(rows) if d is None else np.abs(np64(d))
    none = ((t < 0) | (t >= V)).numpy()
    e = 2 * logit_error(x, w) + 2.0 ** -19 + (64 + V / 128) * 2.0 ** -23 + 2.0 ** -22 * np.abs(np64(lse))
    p = np.abs(P) + np.where(none, 0, scale)[:, None] * (np.arange(V)[None, :] == t.numpy()[:, None])      # the softmax itself, at most
    eP = HALF * np.abs(P) + (1 + HALF) * e[:, None] * p + 2.0 ** -126
    aP, X, W = np.abs(P) + eP, np.abs(np64(x)), np.abs(np64(w))
    # (dx: its fp32 sum over the vocabulary also goes through memory once per piece)
    near(got[0], dx, HALF * np.abs(dx) + (1 + HALF) * (eP @ W + 2 * acc(V) * (aP @ W)) + 2.0 ** -126, "dx")
    near(got[1], dw, HALF * np.abs(dw) + (1 + HALF) * (eP.T @ X + acc(rows) * (aP.T @ X)) + 2.0 ** -126, "dw")
    assert not got[0].cpu()[torch.from_numpy(none)].any()


def test_vocab_loss_in_several_pieces_of_the_vocabulary():
    """Rows enough that the gradient takes the vocabulary in pieces (fp32 sums of dx between them); some rows of each against the oracle."""
    rows, D, V = 16384, 64, 20011
    x, w, t, d = make_loss(rows, D, V, seed=77)
    xd, wd, td, dd = dev(x, w, t, d)
    loss, lse = gf.vocab_loss(xd, wd, td)
    before = gf.launch_count()
    dx, dw = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    assert gf.launch_count() - before in (6, 9)      # three pieces of 6912 columns at most, two kernels each or three
    pick = torch.cat([torch.arange(0, rows, 173), torch.tensor([rows - 1])])
    want, _, P = orc.vocab_loss_backward(x[pick], w, t[pick], d[pick])
    e = 2 * logit_error(x[pick], w)[:, None] + 2.0 ** -18
    eP = HALF * np.abs(P) + (1 + HALF) * e * (np.abs(P) + np.abs(np64(d[pick]))[:, None] * (np.arange(V)[None, :] == t[pick].numpy()[:, None]))
    W = np.abs(np64(w))
    near(dx.cpu()[pick], want, HALF * np.abs(want) + (1 + HALF) * (eP @ W + 2 * acc(V) * ((np.abs(P) + eP) @ W)) + 2.0 ** -126, "dx")
    # dw: all rows count, so columns of the vocabulary around the pieces' edges, in float64 on the device
    cols = torch.tensor([0, 1, 6911, 6912, 6913, 13823, 13824, 20009, 20010], device=DEV)
    z = xd.double() @ wd[cols].double().t() - lse.double()[:, None]
    has = (td >= 0) & (td < V)
    Pc = (z.exp() - (td[:, None] == cols[None, :]).double()) * (dd.double() * has)[:, None]
    want = Pc.t() @ xd.double()
    e = (HALF + 2.0 ** -14 + acc(rows)) * (Pc.abs() + (td[:, None] == cols[None, :]) * dd.abs()[:, None]).t() @ xd.double().abs()
    near(dw[cols], np64(want), HALF * np.abs(np64(want)) + (1 + HALF) * np64(e), "dw")


def test_vocab_loss_of_large_and_infinite_logits_and_of_nothing():
    D, V = 64, 300
    w = torch.zeros(V, D)
    w[:, 0] = torch.linspace(-1, 1, V)
    w[7, 1] = 1.0
    x = torch.zeros(5, D)
    x[0, 0] = 30000.0                                # exp of the logits themselves would overflow
    x[1, 0] = -30000.0
    x[2, 1] = float("inf")                           # 0 * inf: NaN in every other logit
    t = torch.tensor([V - 1, 0, 7, 5, -100])
    x, w = x.to(BF), w.to(BF)
    xd, wd, td = dev(x, w, t)
    loss, lse = gf.vocab_loss(xd, wd, td)
    gf.last_device_status()
    want, want_lse = orc.vocab_loss(x[[0, 1, 3, 4]], w, t[[0, 1, 3, 4]])
    near(lse[[0, 1, 3, 4]], want_lse, 2.0 ** -20 * (1 + np.abs(want_lse)), "lse")
    near(loss[[0, 1, 3, 4]], want, 2.0 ** -20 * (1 + np.abs(want_lse)), "loss")
    assert torch.isnan(lse[2]) and torch.isnan(loss[2]) and loss[4] == 0
    clean = torch.tensor([0, 1, 3, 4], device=DEV)
    dx, _ = gf.vocab_loss_backward(xd, wd, td, lse)
    assert torch.isnan(dx[2]).any() and torch.isfinite(dx[clean]).all() and not dx[4].any()
    none, no_t = torch.empty(0, D, dtype=BF, device=DEV), torch.empty(0, dtype=torch.int64, device=DEV)
    loss, lse = gf.vocab_loss(none, wd, no_t)
    dx, dw = gf.vocab_loss_backward(none, wd, no_t, lse)
    assert loss.shape == lse.shape == (0,) and dx.shape == (0, D) and not dw.any()


def test_vocab_loss_of_next_tokens_and_rows_without_a_target():
    """Labels that are the tokens from the second one on (aligned to 8 bytes only), losses' weights that start anywhere, and a row without a
    target whose logits overflow: nothing of it reaches the gradients."""
    g = torch.Generator().manual_seed(6)
    ids = torch.randint(0, 300, (129,), generator=g).to(DEV)
    x, w = dev(normal(g, 129, 64), normal(g, 300, 64))
    d = torch.randn(130, generator=g).to(DEV)
    got = gf.vocab_loss(x[:-1], w, ids[1:])
    want = gf.vocab_loss(x[:-1], w, ids[1:].clone())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    lse = torch.cat([torch.zeros(1, device=DEV), got[1]])[1:]
    a, b = gf.vocab_loss_backward(x[:-1], w, ids[1:], lse, d[1:129]), gf.vocab_loss_backward(x[:-1], w, ids[1:].clone(), got[1], d[1:129].clone())
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    t = ids.clone()
    t[5] = -100
    loss, lse = gf.vocab_loss(x, w, t)
    clean = gf.vocab_loss_backward(x, w, t, lse)
    lse[5] = float("nan")
    got = gf.vocab_loss_backward(x, w, t, lse)
    gf.last_device_status()
    assert all(torch.equal(p, q) for p, q in zip(got, clean)) and not got[0][5].any()


# ------------------------------------------------------------------------------------------------ as they are used together
class Block:
    """The end of a Finch-C2 block, the channel mix and the loss, forward and backward, as a training step runs them."""

    def __init__(self, T=300, H=4, V=1003, seed=1):
        g = torch.Generator().manual_seed(seed)
        D = 64 * H
        F = 7 * D // 2
        self.H = H
        self.y = normal(g, T, H, 64, std=2).to(DEV)
        self.gamma = (1 + normal(g, D, std=0.3, dtype=torch.float32)).to(DEV)
        self.wk, self.wv, self.wr = (normal(g, a, b, std=a ** -0.5).to(DEV) for a, b in ((D, F), (F, D), (D, D)))
        self.head = normal(g, V, D, std=2 * D ** -0.5).to(DEV)
        self.t = torch.randint(0, V, (T,), generator=g).to(DEV)
        self.d = torch.full((T,), 1.0 / T, device=DEV)

    def step(self, sync=lambda: None):
        o = {}
        o["n"] = gf.layernorm_heads(self.y, self.gamma).flatten(1); sync()
        o["h"] = gf.gated_linear(o["n"], self.wk, act="relu2"); sync()
        o["o"] = gf.gated_linear(o["n"], self.wr, o["h"], self.wv, act="sigmoid"); sync()
        o["loss"], o["lse"] = gf.vocab_loss(o["o"], self.head, self.t); sync()
        o["do"], o["dhead"] = gf.vocab_loss_backward(o["o"], self.head, self.t, o["lse"], self.d); sync()
        o["dn1"], o["dwr"], o["dh"], o["dwv"] = gf.gated_linear_backward(o["n"], self.wr, o["do"], o["h"], self.wv, act="sigmoid"); sync()
        o["dn2"], o["dwk"], _, _ = gf.gated_linear_backward(o["n"], self.wk, o["dh"], act="relu2"); sync()
        o["dn"] = o["dn1"] + o["dn2"]
        o["dy"], o["dgamma"], _ = gf.layernorm_heads_backward(self.y, o["dn"].view_as(self.y), self.gamma); sync()
        return o


def test_training_step_through_the_operators_matches_float64_step_by_step():
    """Every operator of the run against the oracle on the inputs it had, and the run's gradients against automatic differentiation of the
    whole in float64: at most nine values in a row are rounded to bf16 on the way to any of them."""
    b = Block()
    o = b.step()
    gf.last_device_status()
    check_gate(o["n"], b.wk, None, None, "relu2", o["h"], "h")
    check_gate(o["n"], b.wr, o["h"], b.wv, "sigmoid", o["o"], "o")
    check_gate_grad(o["n"], b.wr, o["h"], b.wv, "sigmoid", o["do"], (o["dn1"], o["dwr"], o["dh"], o["dwv"]), "gate")
    check_gate_grad(o["n"], b.wk, None, None, "relu2", o["dh"], (o["dn2"], o["dwk"], None, None), "hidden")
    check_norm(b.y, o["dn"].view_as(b.y), b.gamma, 1e-5, (o["dy"], o["dgamma"], o["dn"].double().sum(0)), "norm")
    y, gamma, wk, wv, wr, head = (t.double().requires_grad_() for t in (b.y, b.gamma, b.wk, b.wv, b.wr, b.head))
    n = torch.nn.functional.layer_norm(y.flatten(1), (64 * b.H,), gamma, None, 1e-5)
    out = torch.sigmoid(n @ wr) * (torch.relu(n @ wk).square() @ wv)
    loss = torch.nn.functional.cross_entropy(out @ head.t(), b.t, reduction="none")
    grads = torch.autograd.grad((loss * b.d).sum(), (y, gamma, wk, wv, wr, head))
    assert (o["loss"].double() - loss).norm() <= 9 * HALF * loss.norm()
    for name, g in zip(("dy", "dgamma", "dwk", "dwv", "dwr", "dhead"), grads):
        e = ((o[name].double() - g).norm() / g.norm()).item()
        assert e <= 9 * HALF, (name, e)


@pytest.mark.parametrize("rows", [1, 5, 128])
def test_gradients_of_few_rows_are_off_by_their_own_rounding_alone(rows):
    """Of up to 128 rows da, db and P are kept to 16 bits of mantissa (a rounding and what it leaves, each off by HALF of itself), so every element
    of a gradient is off by its rounding, HALF, and HALF^2 of the magnitudes it is the sum of."""
    x, w, x2, w2, dy = make_gate(rows, 136, 72, 264, seed=rows)
    got = gf.gated_linear_backward(*dev(x, w, dy, x2, w2), act="silu")
    want = orc.gated_linear_backward(x, w, dy, x2, w2, act="silu")
    a, ea, b, eb, f, ef, df, edf = gate_parts(x, w, x2, w2, "silu")
    d = np.abs(np64(dy))
    da, db = d * np.abs(b) * np.abs(df), d * np.abs(f)
    eda, edb = HALF ** 2 * da + d * (edf * (np.abs(b) + eb) + np.abs(df) * eb), HALF ** 2 * db + d * ef
    X, W, X2, W2 = (np.abs(np64(t)) for t in (x, w, x2, w2))
    n = 2 * acc(264)
    bounds = [eda @ W.T + n * (da @ W.T), X.T @ eda + n * (X.T @ da), edb @ W2.T + n * (db @ W2.T), X2.T @ edb + n * (X2.T @ db)]
    for name, g, t, e in zip(("dx", "dw", "dx2", "dw2"), got, want, bounds):
        near(g, t, HALF * np.abs(t) + (1 + HALF) * e + 2.0 ** -126, name)
    x, w, t, dl = make_loss(rows, 136, 1003, seed=rows)
    xd, wd, td, dd = dev(x, w, t, dl)
    lse = gf.vocab_loss(xd, wd, td)[1]
    got = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    dx, dw, P = orc.vocab_loss_backward(x, w, t, dl)
    e = 2 * logit_error(x, w) + 2.0 ** -19 + (64 + 1003 / 128) * 2.0 ** -23 + 2.0 ** -22 * np.abs(np64(lse))
    has = ((t >= 0) & (t < 1003)).numpy()
    p = np.abs(P) + np.where(has, np.abs(np64(dl)), 0)[:, None] * (np.arange(1003)[None, :] == t.numpy()[:, None])
    eP, X, W = (HALF ** 2 + e[:, None]) * p, np.abs(np64(x)), np.abs(np64(w))
    n = 2 * acc(2 * 1003)
    near(got[0], dx, HALF * np.abs(dx) + (1 + HALF) * (eP @ W + n * (np.abs(P) @ W)) + 2.0 ** -126, "dx")
    near(got[1], dw, HALF * np.abs(dw) + (1 + HALF) * (eP.T @ X + n * (np.abs(P).T @ X)) + 2.0 ** -126, "dw")


def test_training_step_back_to_back_equals_one_call_at_a_time():
    b = Block(T=1111, H=12, V=4001)
    one = b.step(torch.cuda.synchronize)
    runs = [b.step() for _ in range(3)]
    torch.cuda.synchronize()
    gf.last_device_status()
    for r in runs:
        for k in one:
            assert torch.equal(r[k], one[k]), k


def test_training_step_captured_and_replayed_on_new_inputs():
    b, other = Block(T=500), Block(T=500, seed=2)
    want = other.step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = b.step()
    for n in ("y", "gamma", "wk", "wv", "wr", "head", "t", "d"):
        getattr(b, n).copy_(getattr(other, n))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    gf.last_device_status()
    for k in want:
        assert torch.equal(out[k], want[k]), k


def test_calls_on_another_stream_and_two_at_a_time():
    """The same calls on two streams at once, each with its own workspace from the caching allocator."""
    blocks = [Block(T=700, H=8, V=3001, seed=s) for s in (1, 2)]
    want = [b.step() for b in blocks]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in blocks]
    got = [None, None]
    for i, (b, s) in enumerate(zip(blocks, streams)):
        with torch.cuda.stream(s):
            got[i] = [b.step() for _ in range(3)][-1]
    torch.cuda.synchronize()
    gf.last_device_status()
    for g, w in zip(got, want):
        for k in w:
            assert torch.equal(g[k], w[k]), k


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 bytes and 2^31 elements: rows at both ends against the same rows by themselves."""
    rows, D, V = 1_100_000, 2048, 300
    ends = torch.cat([torch.arange(128), torch.arange(rows - 128, rows)]).to(DEV)
    g = torch.Generator(device=DEV).manual_seed(5)
    block = torch.randn(1000, D, generator=g, device=DEV).to(BF)
    y = block.repeat(rows // 1000, 1)
    dout = y.flip(1)
    dy = gf.layernorm_heads_backward(y.view(rows, 32, 64), dout.view(rows, 32, 64), want_params=False)[0].view(rows, D)
    few = gf.layernorm_heads_backward(y[ends].view(-1, 32, 64), dout[ends].view(-1, 32, 64), want_params=False)[0].view(-1, D)
    assert torch.equal(dy[ends], few) and torch.equal(dy[-1000:], dy[:1000])
    del dy, dout
    w, x = torch.randn(64, D, generator=g, device=DEV).to(BF) / 8, y[:, :64].contiguous()
    out = gf.gated_linear(x, w, act="sigmoid")
    want = gf.gated_linear(x[ends].contiguous(), w, act="sigmoid")
    assert_near(out[ends], want)
    dx = gf.gated_linear_backward(x, w, y, act="sigmoid")[0]
    assert_near(dx[ends], gf.gated_linear_backward(x[ends].contiguous(), w, y[ends], act="sigmoid")[0])
    del out, y
    t = torch.randint(0, V, (rows,), generator=g, device=DEV)
    head = torch.randn(V, 64, generator=g, device=DEV).to(BF)
    loss, lse = gf.vocab_loss(x, head, t)
    few = gf.vocab_loss(x[ends].contiguous(), head, t[ends])
    assert (loss[ends] - few[0]).abs().max() < 1e-4
    dx = gf.vocab_loss_backward(x, head, t, lse)[0]
    assert_near(dx[ends], gf.vocab_loss_backward(x[ends].contiguous(), head, t[ends], few[1])[0])
    gf.last_device_status()


def assert_near(a, b):
    """The same rows through tiles of another shape: an operand and the result rounded to bf16 once each, from sums in another order."""
    a, b = a.double(), b.double()
    assert (a - b).norm() <= 2 * HALF * b.norm() and torch.isfinite(a).all()


def test_binding_checks_shapes_and_types():
    x, w, x2, w2, dy = dev(*make_gate(16, 64, 72, 136, seed=1))
    for bad in (lambda: gf.gated_linear(x, w, x, w2), lambda: gf.gated_linear(x.float(), w), lambda: gf.gated_linear(x.t().contiguous().t(), w),
                lambda: gf.gated_linear(x, w, x2[:8], w2), lambda: gf.gated_linear_backward(x, w, dy[:, :64].contiguous()),
                lambda: gf.gated_linear(x, w, out=torch.empty(16, 72, dtype=BF, device=DEV)), lambda: gf.vocab_loss(x, w2, torch.zeros(16, dtype=torch.int64, device=DEV)),
                lambda: gf.vocab_loss(x, w.t().contiguous(), torch.zeros(16, dtype=torch.int32, device=DEV)),
                lambda: gf.layernorm_heads_backward(dy.view(16, 2, 68), dy.view(16, 68, 2)), lambda: gf.vocab_loss(x, w.t().contiguous(), torch.zeros(16, dtype=torch.int64))):
        with pytest.raises((ValueError, TypeError)):
            bad()
