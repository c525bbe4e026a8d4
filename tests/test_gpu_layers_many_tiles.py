"""The operators around the recurrence where a CTA, or a pair of them, goes through several tiles or stages: accumulators, barriers and slabs in their
second and later use, column sums carried over stages, fp32 sums of one piece taken up by the next.  That the shapes do this is asserted without a
GPU in test_host_layer_tiles.py.  Bounds as in test_gpu_layers.py, in float64 on the GPU where the sizes are large."""
import numpy as np
import pytest
import torch

import paper_2407_12077_b200 as gf
from oracle import wkv6_oracle as orc
from test_gpu_layers import (ACTS, BF, CANARY, DEV, HALF, acc, check_gate, check_gate_grad, dev, gate_parts, logit_error, make_gate, make_loss, near, normal,
                             np64)

pytestmark = pytest.mark.gpu

# two products of their own depth, each with a whole accumulator of its own: two and three tiles to a pair, the last rows and columns ragged (4000: a
# block of 32 columns at the end; 6008: the second CTA of the last pair has no column, of the last band of 2100 rows no row)
WIDE = [(2300, 264, 328, 4000), (2100, 264, 328, 6008)]
# (more than one tile per CTA, up to 128 rows: products of few rows keep what rounding leaves of their first operands)
FEW_GATE = [(5, 72, 136, 10008), (128, 136, 0, 10008), (100, 64, -1, 20008)]
FEW_LOSS = [(5, 64, 40011), (128, 136, 40011)]


@pytest.mark.parametrize("rows,K1,K2,F", WIDE)
@pytest.mark.parametrize("act", ACTS)
def test_gated_linear_over_several_wide_tiles(rows, K1, K2, F, act):
    x, w, x2, w2, dy = make_gate(rows, K1, K2, F, seed=rows + F)
    room = torch.full((rows + 2, F), CANARY, dtype=BF, device=DEV)
    gf.gated_linear(*dev(x, w, x2, w2), act=act, out=room[1:rows + 1])
    gf.last_device_status()
    assert torch.all(room[0] == CANARY) and torch.all(room[-1] == CANARY)
    check_gate(x, w, x2, w2, act, room[1:rows + 1], f"{rows} {K1} {K2} {F} {act}")
    got = gf.gated_linear_backward(*dev(x, w, dy, x2, w2), act=act)
    gf.last_device_status()
    check_gate_grad(x, w, x2, w2, act, dy, got, f"{rows} {K1} {K2} {F} {act}")


@pytest.mark.parametrize("rows,K1,K2,F", FEW_GATE)
@pytest.mark.parametrize("act", ["silu", "relu2"])
def test_gate_gradient_of_few_rows_over_several_tiles(rows, K1, K2, F, act):
    x, w, x2, w2, dy = make_gate(rows, K1, K2, F, seed=rows + F)
    got = gf.gated_linear_backward(*dev(x, w, dy, x2, w2), act=act)
    gf.last_device_status()
    check_gate_grad(x, w, x2, w2, act, dy, got, f"{rows} {K1} {K2} {F} {act}")
    # and closer: da and db are kept to HALF^2
    a, ea, b, eb, f, ef, df, edf = gate_parts(x, w, x2, w2, act)
    d = np.abs(np64(dy))
    da = d * np.abs(b) * np.abs(df)
    eda = HALF ** 2 * da + d * (edf * (np.abs(b) + eb) + np.abs(df) * eb)
    X = np.abs(np64(x))
    want = orc.gated_linear_backward(x, w, dy, x2, w2, act=act)[1]
    near(got[1], want, HALF * np.abs(want) + (1 + HALF) * (X.T @ eda + 2 * acc(rows) * (X.T @ da)) + 2.0 ** -126, "dw")


@pytest.mark.parametrize("rows,D,V", FEW_LOSS)
def test_loss_gradient_of_few_rows_over_several_tiles(rows, D, V):
    x, w, t, dl = make_loss(rows, D, V, seed=rows)
    xd, wd, td, dd = dev(x, w, t, dl)
    loss, lse = gf.vocab_loss(xd, wd, td)
    got = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    want, want_lse = orc.vocab_loss(x, w, t)
    e = logit_error(x, w) + 2.0 ** -20 + (64 + V / 128) * 2.0 ** -23
    near(lse, want_lse, e + 2.0 ** -23 * np.abs(want_lse), "lse")
    near(loss, want, 2 * e + 2.0 ** -22 * (np.abs(want_lse) + np.abs(want)), "loss")
    dx, dw, P = orc.vocab_loss_backward(x, w, t, dl)
    e = 2 * logit_error(x, w) + 2.0 ** -19 + (64 + V / 128) * 2.0 ** -23 + 2.0 ** -22 * np.abs(np64(lse))
    has = ((t >= 0) & (t < V)).numpy()
    p = np.abs(P) + np.where(has, np.abs(np64(dl)), 0)[:, None] * (np.arange(V)[None, :] == t.numpy()[:, None])
    eP, X, W = (HALF ** 2 + e[:, None]) * p, np.abs(np64(x)), np.abs(np64(w))
    near(got[0], dx, HALF * np.abs(dx) + (1 + HALF) * (eP @ W + 2 * acc(2 * V) * (np.abs(P) @ W)) + 2.0 ** -126, "dx")
    near(got[1], dw, HALF * np.abs(dw) + (1 + HALF) * (eP.T @ X + 2 * acc(2 * rows) * (np.abs(P).T @ X)) + 2.0 ** -126, "dw")


def test_loss_gradient_whose_sum_over_the_pieces_is_not_cut():
    """Two pieces of the vocabulary, dx's tiles enough that they are not cut along the contraction index: the first piece's fp32 sums are taken up in the
    second one's epilogue.  Everything in float64 on the GPU."""
    rows, D, V = 16384, 1024, 8200
    x, w, t, d = make_loss(rows, D, V, seed=5)
    xd, wd, td, dd = dev(x, w, t, d)
    loss, lse = gf.vocab_loss(xd, wd, td)
    before = gf.launch_count()
    dx, dw = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    assert gf.launch_count() - before == 4
    X, W = xd.double(), wd.double()
    z = X @ W.t()
    want_lse = torch.logsumexp(z, 1)
    e = (acc(D) * (X.abs() @ W.abs().t()).amax(1)) + 2.0 ** -20 + (64 + V / 128) * 2.0 ** -23
    assert ((lse.double() - want_lse).abs() <= e + 2.0 ** -23 * want_lse.abs()).all()
    has = ((td >= 0) & (td < V)).double()
    weight = (dd.double() * has)[:, None]
    hot = torch.zeros_like(z)
    hot[torch.arange(rows, device=DEV), td.clamp(0, V - 1)] = 1
    p = (z - want_lse[:, None]).exp_()
    del z
    P, size = (p - hot) * weight, (p + hot) * weight.abs()
    del p, hot
    eP = HALF * P.abs() + (1 + HALF) * (2 * e + 2.0 ** -19 + 2.0 ** -22 * want_lse.abs())[:, None] * size + 2.0 ** -126
    aP = P.abs() + eP
    for name, got, want, bound in (("dx", dx, P @ W, eP @ W.abs() + 2 * acc(V) * (aP @ W.abs())), ("dw", dw, P.t() @ X, eP.t() @ X.abs() + acc(rows) * (aP.t() @ X.abs()))):
        off = (got.double() - want).abs() - (HALF * want.abs() + (1 + HALF) * bound + 2.0 ** -126)
        assert not (off > 0).any() and torch.isfinite(got).all(), (name, int((off > 0).sum()), float(off.max()))


# every variant of the norm's gradient (units of 16 bytes in a row), and rows enough for five stages to a CTA and a ragged last one
NORM = [(BF, 1, 64), (BF, 4, 64), (BF, 8, 64), (BF, 12, 64), (BF, 16, 64), (BF, 65, 8), (BF, 32, 64), (BF, 64, 64), (BF, 128, 64),
        (torch.float32, 1, 64), (torch.float32, 4, 64), (torch.float32, 6, 64), (torch.float32, 8, 64), (torch.float32, 16, 64), (torch.float32, 32, 64),
        (torch.float32, 64, 64), (torch.float32, 128, 64)]


def norm_rows(dtype, H, N):
    return 26_000_000 // (H * N * torch.finfo(dtype).bits // 8) | 1


def norm_reference(y, dout, gamma, eps):
    """Of one block of rows, in float64: (dy, the sizes of its terms, dgamma, dbeta, and the sums of the magnitudes of both)."""
    y, dout, gm = y.double().flatten(1), dout.double().flatten(1), gamma.double()
    c = y - y.mean(1, keepdim=True)
    rstd = (c.square().mean(1, keepdim=True) + eps).rsqrt()
    xhat, g = c * rstd, dout * gm
    dy = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    terms = rstd * (g.abs() + g.abs().mean(1, keepdim=True) + xhat.abs() * (g * xhat).abs().mean(1, keepdim=True))
    # the mean is rounded, after a butterfly and a lane's run of additions: 40 steps of the largest magnitude, and with it every deviation
    off = y.abs().amax(1, keepdim=True) * rstd
    terms = terms + rstd * off * ((g * xhat).abs().mean(1, keepdim=True) + xhat.abs() * g.abs().mean(1, keepdim=True))
    size = dout.abs() * (xhat.abs() + off)
    return dy, terms, (dout * xhat).sum(0), dout.sum(0), size.sum(0), dout.abs().sum(0), size.square().sum(0)


@pytest.mark.parametrize("dtype,H,N", NORM)
def test_norm_gradient_over_many_stages(dtype, H, N):
    rows, D = norm_rows(dtype, H, N), H * N
    g = torch.Generator(device=DEV).manual_seed(H)
    y = (torch.randn(rows, H, N, generator=g, device=DEV) * 2 + 0.3).to(dtype)
    dout = torch.randn(rows, H, N, generator=g, device=DEV).to(dtype)
    gamma = 1 + 0.5 * torch.randn(D, generator=g, device=DEV)
    dy, dgamma, dbeta = gf.layernorm_heads_backward(y, dout, gamma, 1e-5)
    gf.last_device_status()
    u = 40 * 2.0 ** -23
    sums = [torch.zeros(D, dtype=torch.float64, device=DEV) for _ in range(4)]
    step = max(1, 16_000_000 // D)
    for i in range(0, rows, step):
        want, terms, *s = norm_reference(y[i:i + step], dout[i:i + step], gamma, 1e-5)
        off = (dy[i:i + step].double().flatten(1) - want).abs() - (u * terms + (HALF if dtype == BF else 2.0 ** -24) * want.abs())
        assert not (off > 0).any(), (i, float(off.max()))
        for a, b in zip(sums, s):
            a += b
    # a column's sum: additions of a thread's rows (at most rows / 148 of them), of 64 groups and of 64 again, each off by half a step of the sum of magnitudes
    n = (rows / 148 + 200) * 2.0 ** -24
    assert ((dgamma.double() - sums[0]).abs() <= (u + n) * sums[2]).all()
    assert ((dbeta.double() - sums[1]).abs() <= n * sums[3]).all()


@pytest.mark.parametrize("dtype,H,N", NORM)
def test_norm_gradient_counts_every_row_once(dtype, H, N):
    """y and dout of +-1 with as many of either in a row: mean 0, variance 1 (eps 0), xhat = y, so dbeta is a sum of whole numbers below 2^24, exact, and
    dgamma one of +-1 off by some steps each (under 2^-18 of rows, below 0.4): a row left out, or taken twice, changes every column by one."""
    rows, D = norm_rows(dtype, H, N), H * N
    g = torch.Generator(device=DEV).manual_seed(H + 1)
    half = torch.ones(D, device=DEV)
    half[::2] = -1
    sign = torch.randint(0, 2, (rows, 1), generator=g, device=DEV) * 2.0 - 1
    y = (sign * half).to(dtype).view(rows, H, N)
    dout = (torch.randint(0, 2, (rows, D), generator=g, device=DEV) * 2 - 1).to(dtype).view(rows, H, N)
    _, dgamma, dbeta = gf.layernorm_heads_backward(y, dout, None, 0.0)
    gf.last_device_status()
    assert torch.equal(dbeta.double(), dout.flatten(1).sum(0, dtype=torch.float64))
    assert ((dgamma.double() - (dout.double() * y.double()).flatten(1).sum(0)).abs() <= 0.45).all()


@pytest.mark.parametrize("rows,targets", [(129, 1), (129, 5), (2048, 1), (2048, 5)])
def test_gradients_of_a_batch_that_is_masked_but_for_a_few_rows(rows, targets):
    """P is kept in bf16 of more than 128 rows, however few of them have a target: HALF of its own magnitude each, and the result's HALF."""
    D, V = 136, 1003
    x, w, _, d = make_loss(rows, D, V, seed=rows)
    t = torch.full((rows,), -100)
    at = torch.arange(targets) * (rows // targets)
    t[at] = torch.arange(targets) * 7
    xd, wd, td, dd = dev(x, w, t, d)
    lse = gf.vocab_loss(xd, wd, td)[1]
    got = gf.vocab_loss_backward(xd, wd, td, lse, dd)
    gf.last_device_status()
    dx, dw, P = orc.vocab_loss_backward(x, w, t, d)
    e = 2 * logit_error(x, w) + 2.0 ** -19 + (64 + V / 128) * 2.0 ** -23 + 2.0 ** -22 * np.abs(np64(lse))
    has = (t >= 0).numpy()
    p = np.abs(P) + np.where(has, np.abs(np64(d)), 0)[:, None] * (np.arange(V)[None, :] == t.numpy()[:, None])
    eP = HALF * np.abs(P) + (1 + HALF) * e[:, None] * p
    aP, X, W = np.abs(P) + eP, np.abs(np64(x)), np.abs(np64(w))
    near(got[0], dx, HALF * np.abs(dx) + (1 + HALF) * (eP @ W + 2 * acc(V) * (aP @ W)) + 2.0 ** -126, "dx")
    near(got[1], dw, HALF * np.abs(dw) + (1 + HALF) * (eP.T @ X + acc(rows) * (aP.T @ X)) + 2.0 ** -126, "dw")
    assert not got[0].cpu()[torch.from_numpy(~has)].any()
