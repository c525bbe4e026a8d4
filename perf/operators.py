"""The operators around the recurrence in a training or serving step, as a program built on this library calls them: the
gradient of the LayerNorm across all heads, the gated linear block of the channel mix with its gradient, and the
cross entropy over the vocabulary with its gradient.

Sizes are those of the D = 768 and D = 2048 models of the benchmark configurations (hidden width 3.5 D in the channel
mix) or generic ones beside them.  Activations are of unit variance, weights keep it, as behind a normalisation.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # gradient of the norm behind the recurrence: one short prompt's fine-tuning step in the D = 768 model, where latency counts
        dict(name="norm-grad-prompt", kind="norm_grad", dtype="bf16", rows=333, H=12),
        # the training batch of 8 sequences of 2048 tokens in the D = 2048 model
        dict(name="norm-grad-train", kind="norm_grad", dtype="bf16", rows=16384, H=32),
        # everything in fp32 and wider, rows that divide by nothing
        dict(name="norm-grad-fp32", kind="norm_grad", dtype="f32", rows=10007, H=64),
        # decode: the gate that ends the D = 2048 channel mix, sigmoid(x_r W_r) * (h W_v), for four sequences' next tokens
        dict(name="gate-decode", kind="gate", act="sigmoid", rows=4, K1=2048, K2=7168, F=2048),
        # one prompt through a gated hidden layer of the D = 768 model, both products of the same input
        dict(name="gate-prompt", kind="gate", act="silu", rows=333, K1=768, K2=0, F=2688),
        # the same gate as in decode over a training batch
        dict(name="gate-train", kind="gate", act="sigmoid", rows=16384, K1=2048, K2=7168, F=2048),
        # gradient of the hidden layer of the D = 768 channel mix, relu(x W)^2, over a ragged small batch
        dict(name="gate-grad-small", kind="gate_grad", act="relu2", rows=1111, K1=768, K2=-1, F=2688),
        # gradient of a gated hidden layer of the D = 2048 model, both products of the same input, over half a training batch
        dict(name="gate-grad-train", kind="gate_grad", act="silu", rows=8192, K1=2048, K2=0, F=7168),
        # scoring a few tokens against an odd vocabulary with the D = 768 model
        dict(name="loss-few", kind="loss", rows=7, D=768, V=40011),
        # validation loss of a long document with the D = 2048 model
        dict(name="loss-document", kind="loss", rows=8192, D=2048, V=65536),
        # a ragged fine-tuning batch of the D = 768 model: the loss and its gradients
        dict(name="loss-grad-small", kind="loss_grad", rows=1500, D=768, V=40011),
        # the training batch's loss and gradients, four sequences of 2048 tokens
        dict(name="loss-grad-train", kind="loss_grad", rows=8192, D=2048, V=65536),
    ]


def _log(rng, lo, hi):
    """A whole number from lo..hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm_grad", "gate", "gate", "gate_grad", "loss", "loss_grad"])
    if kind == "norm_grad":
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), rows=_log(rng, 1, 16384), H=rng.choice([1, 4, 12, 20, 32, 40, 64, 128]))
    if kind in ("gate", "gate_grad"):
        K1 = 8 * _log(rng, 8, 256)
        F = 8 * _log(rng, 8, 896)
        # K2 = 0: both products of one input; -1: no second product
        K2 = rng.choice([0, 0, -1, 8 * _log(rng, 8, 896)])
        return dict(kind=kind, act=rng.choice(["sigmoid", "silu", "relu2", "gelu"]), rows=_log(rng, 1, 16384 if kind == "gate" else 8192), K1=K1, K2=K2, F=F)
    return dict(kind=kind, rows=_log(rng, 1, 8192), D=8 * _log(rng, 16, 256), V=_log(rng, 500, 65536))


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)

    kind = case["kind"]
    s = dict(case)
    if kind == "norm_grad":
        rows, H, dt = case["rows"], case["H"], TYPES[case["dtype"]]
        s.update(y=normal(rows, H, 64, dtype=dt), dout=normal(rows, H, 64, dtype=dt), eps=1e-5,
                 gamma=1 + normal(H * 64, std=0.3, dtype=torch.float32))
    elif kind in ("gate", "gate_grad"):
        rows, K1, K2, F = (case[n] for n in ("rows", "K1", "K2", "F"))
        s.update(x=normal(rows, K1), w=normal(K1, F, std=K1 ** -0.5), x2=None, w2=None)
        if K2 >= 0:
            s["w2"] = normal(K2 or K1, F, std=(K2 or K1) ** -0.5)
        if K2 > 0:
            s["x2"] = normal(rows, K2)
        if kind == "gate_grad":
            s["dy"] = normal(rows, F)
    else:
        rows, D, V = (case[n] for n in ("rows", "D", "V"))
        # logits of standard deviation 2; one row in sixteen has no target
        s.update(x=normal(rows, D), w=normal(V, D, std=2 * D ** -0.5),
                 targets=torch.randint(0, V, (rows,), generator=g, device=DEV))
        s["targets"][torch.rand(rows, generator=g, device=DEV) < 1 / 16] = -100
        if kind == "loss_grad":
            s["dloss"] = (0.5 + torch.rand(rows, generator=g, device=DEV)) / rows
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    import paper_2407_12077_b200 as gf

    kind = s["kind"]
    if kind == "norm_grad":
        return gf.layernorm_heads_backward(s["y"], s["dout"], s["gamma"], s["eps"])
    if kind == "gate":
        return gf.gated_linear(s["x"], s["w"], s["x2"], s["w2"], act=s["act"])
    if kind == "gate_grad":
        return gf.gated_linear_backward(s["x"], s["w"], s["dy"], s["x2"], s["w2"], act=s["act"])
    loss, lse = gf.vocab_loss(s["x"], s["w"], s["targets"])
    if kind == "loss":
        return loss, lse
    return (loss, lse) + tuple(gf.vocab_loss_backward(s["x"], s["w"], s["targets"], lse, s["dloss"]))


def _plain(s):
    kind = s["kind"]
    if kind == "norm_grad":
        y, dout = s["y"].float().flatten(1), s["dout"].float().flatten(1)
        c = y - y.mean(1, keepdim=True)
        rstd = (c.square().mean(1, keepdim=True) + s["eps"]).rsqrt()
        xhat, gd = c * rstd, dout * s["gamma"]
        dy = rstd * (gd - gd.mean(1, keepdim=True) - xhat * (gd * xhat).mean(1, keepdim=True))
        return dy.to(s["y"].dtype).view_as(s["y"]), (dout * xhat).sum(0), dout.sum(0)
    if kind in ("gate", "gate_grad"):
        bf = torch.bfloat16
        x, w = s["x"].float(), s["w"].float()
        a = x @ w
        f, df = _act(a, s["act"], kind == "gate_grad")
        x2 = w2 = b = None
        if s["w2"] is not None:
            x2, w2 = x if s["x2"] is None else s["x2"].float(), s["w2"].float()
            b = x2 @ w2
        if kind == "gate":
            return (f if b is None else f * b).to(bf)
        dy = s["dy"].float()
        da = dy * df if b is None else dy * b * df
        dx, dw = da @ w.t(), x.t() @ da
        if b is None:
            return dx.to(bf), dw.to(bf), None, None
        db = dy * f
        dx2, dw2 = db @ w2.t(), x2.t() @ db
        if s["x2"] is None:
            return (dx + dx2).to(bf), dw.to(bf), None, dw2.to(bf)
        return dx.to(bf), dw.to(bf), dx2.to(bf), dw2.to(bf)
    x, w, targets = s["x"].float(), s["w"].float(), s["targets"]
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lse = (top + total.log()).squeeze(1)
    has = targets >= 0
    at = targets.clamp(min=0)[:, None]
    loss = torch.where(has, lse - z.gather(1, at).squeeze(1), torch.zeros_like(lse))
    if kind == "loss":
        return loss, lse
    p = e / total
    p.scatter_add_(1, at, -torch.ones_like(lse)[:, None])
    p *= torch.where(has, s["dloss"], torch.zeros_like(lse))[:, None]
    return loss, lse, (p @ w).to(torch.bfloat16), (p.t() @ x).to(torch.bfloat16)


def _act(a, act, grad):
    """The activation of a, and its derivative where asked for."""
    if act == "relu2":
        r = a.clamp(min=0)
        return r * r, 2 * r if grad else None
    if act == "gelu":
        phi = 0.5 * (1 + torch.erf(a * 0.5 ** 0.5))
        return a * phi, phi + a * torch.exp(-0.5 * a * a) * (2 * math.pi) ** -0.5 if grad else None
    sg = 1 / (1 + torch.exp(-a))
    if act == "sigmoid":
        return sg, sg * (1 - sg) if grad else None
    return a * sg, sg * (1 + a * (1 - sg)) if grad else None


def work(case):
    """Each input read once, each output written once; the products that the results cannot be had without (the gradient's calls
    are given no intermediate values, so the products they need of the forward pass count once)."""
    kind = case["kind"]
    if kind == "norm_grad":
        n = case["rows"] * case["H"] * 64
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": 3 * n * size + 3 * case["H"] * 64 * 4, "flops": 12 * n}
    if kind in ("gate", "gate_grad"):
        rows, K1, K2, F = (case[n] for n in ("rows", "K1", "K2", "F"))
        inputs = rows * (K1 + max(K2, 0))
        depth = K1 + (0 if K2 < 0 else K2 or K1)
        if kind == "gate":
            return {"bytes": 2 * (inputs + depth * F + rows * F), "flops": 2 * rows * F * depth}
        return {"bytes": 2 * (2 * inputs + 2 * depth * F + rows * F), "flops": 6 * rows * F * depth}
    rows, D, V = (case[n] for n in ("rows", "D", "V"))
    if kind == "loss":
        return {"bytes": 2 * (rows * D + V * D) + 16 * rows, "flops": 2 * rows * D * V}
    return {"bytes": 4 * (rows * D + V * D) + 20 * rows, "flops": 6 * rows * D * V}


def exact(case, seed):
    """From the definitions, in 64 bits: gradients by differentiating the operator's formula automatically where that is one
    expression, by the chain rule over blocks of rows where the whole would not fit."""
    s = prepare(case, seed)
    kind = case["kind"]
    d = lambda t: t.detach().double()  # noqa: E731
    if kind == "norm_grad":
        y, gamma = d(s["y"]).flatten(1).requires_grad_(), d(s["gamma"]).requires_grad_()
        beta = torch.zeros_like(gamma, requires_grad=True)
        var, mean = torch.var_mean(y, 1, unbiased=False, keepdim=True)
        out = (y - mean) / torch.sqrt(var + s["eps"]) * gamma + beta
        dy, dgamma, dbeta = torch.autograd.grad(out, (y, gamma, beta), d(s["dout"]).flatten(1))
        return dy.view_as(s["y"]), dgamma, dbeta
    if kind in ("gate", "gate_grad"):
        leaves = [None if s[n] is None else d(s[n]).requires_grad_(kind == "gate_grad") for n in ("x", "w", "x2", "w2")]
        x, w, x2, w2 = leaves
        a = torch.mm(x, w)
        y = {"sigmoid": torch.sigmoid, "silu": lambda t: t * torch.sigmoid(t), "relu2": lambda t: torch.relu(t) ** 2,
             "gelu": lambda t: t * torch.special.ndtr(t)}[case["act"]](a)
        if w2 is not None:
            y = y * torch.mm(x if x2 is None else x2, w2)
        if kind == "gate":
            return y
        asked = [t for t in leaves if t is not None]
        got = iter(torch.autograd.grad(y, asked, d(s["dy"])))
        return tuple(None if t is None else next(got) for t in leaves)
    x, w, targets = d(s["x"]), d(s["w"]), s["targets"]
    loss, lse, dx = [], [], []
    dw = torch.zeros_like(w)
    for i in range(0, x.shape[0], 1024):
        xi, ti = x[i:i + 1024], targets[i:i + 1024]
        logp = torch.mm(xi, w.t())
        li = torch.logsumexp(logp, 1)
        logp -= li[:, None]
        keep = (ti >= 0).nonzero().squeeze(1)
        nll = torch.zeros_like(li)
        nll[keep] = -logp[keep, ti[keep]]
        loss.append(nll)
        lse.append(li)
        if kind == "loss_grad":
            g = logp.exp_()
            g[keep, ti[keep]] -= 1
            weight = torch.zeros_like(li)
            weight[keep] = d(s["dloss"])[i:i + 1024][keep]
            g *= weight[:, None]
            dx.append(torch.mm(g, w))
            dw += torch.mm(g.t(), xi)
    if kind == "loss":
        return torch.cat(loss), torch.cat(lse)
    return torch.cat(loss), torch.cat(lse), torch.cat(dx), dw
