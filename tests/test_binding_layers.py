"""The C++ part of the binding for the operators around the recurrence against the Python code it takes the place of: the same outputs for
the plain form of a call, and for every other form what Python makes of it."""
import pytest
import torch

import paper_2407_12077_b200 as gf

DEV = "cuda:0"
BF = torch.bfloat16


@pytest.fixture
def both(monkeypatch):
    """Runs a call with the C++ part and without it: [result or (exception type, text)] of each."""
    gf.load_library()
    native = gf._native

    def run(fn):
        out = []
        for n in (native, None):
            monkeypatch.setattr(gf, "_native", n)
            try:
                out.append(fn())
            except Exception as e:
                out.append((type(e), str(e)))
        monkeypatch.setattr(gf, "_native", native)
        return out

    return run


def test_leaves_what_is_not_on_the_current_device_to_python():
    gf.load_library()
    if gf._native is None:
        pytest.skip("not built")
    n, t, w, y = gf._native, torch.zeros(4, 64, dtype=BF), torch.zeros(64, 64, dtype=BF), torch.zeros(4, dtype=torch.int64)
    assert n.layernorm_backward(t.view(4, 1, 64), t.view(4, 1, 64), None, 1e-5) is None
    assert n.gated_linear(t, w, None, None, 0) is None and n.gated_linear(t, w, None, None, None) is None
    assert n.gated_linear_backward(t, w, t, None, None, 0) is None
    assert n.vocab_loss(t, w, y) is None and n.vocab_loss_backward(t, w, y, y, None) is None
    for f in (n.layernorm_backward, n.gated_linear, n.gated_linear_backward, n.vocab_loss, n.vocab_loss_backward):
        assert f() is None and f(1, 2, 3, 4, 5, 6) is None


def make():
    g = torch.Generator().manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g).to(DEV).to(BF)  # noqa: E731
    return dict(x=r(2, 35, 64), w=r(64, 136), x2=r(2, 35, 72), w2=r(72, 136), ws=r(64, 136), dy=r(2, 35, 136), head=r(301, 64), y=r(2, 35, 3, 64), dout=r(2, 35, 3, 64),
                t=torch.randint(-1, 301, (2, 35), generator=g).to(DEV), gamma=torch.randn(192, generator=g).to(DEV), d=torch.randn(2, 35, generator=g).to(DEV))


def flat(o):
    return list(o) if isinstance(o, (tuple, list)) else [o]


@pytest.mark.gpu
def test_same_results(both):
    m = make()
    x, w, x2, w2, ws, dy, head, t = (m[n] for n in ("x", "w", "x2", "w2", "ws", "dy", "head", "t"))
    lse = gf.vocab_loss(x, head, t)[1]
    calls = [lambda: gf.layernorm_heads_backward(m["y"], m["dout"], m["gamma"]), lambda: gf.layernorm_heads_backward(m["y"].float(), m["dout"].float(), None, 0.5),
             lambda: gf.layernorm_heads_backward(m["y"], m["dout"], m["gamma"].view(3, 64)),
             lambda: gf.gated_linear(x, w), lambda: gf.gated_linear(x, w, None, ws, act="gelu"), lambda: gf.gated_linear(x, torch.nn.Parameter(w), x2, w2, act="sigmoid"),
             lambda: gf.gated_linear_backward(x, w, dy, act="relu2"), lambda: gf.gated_linear_backward(x, w, dy, None, ws), lambda: gf.gated_linear_backward(x, w, dy, x2, w2),
             lambda: gf.vocab_loss(x, head, t), lambda: gf.vocab_loss(x.clone().requires_grad_(), head, t), lambda: gf.vocab_loss(x[:0], head, t[:0]),
             lambda: gf.vocab_loss_backward(x, head, t, lse), lambda: gf.vocab_loss_backward(x, head, t, lse, m["d"]), lambda: gf.vocab_loss_backward(x[:0], head, t[:0], lse[:0])]
    for n, call in enumerate(calls):
        a, b = both(call)
        assert not (isinstance(a, tuple) and isinstance(a[0], type)), (n, a)
        for p, q in zip(flat(a), flat(b), strict=True):
            assert (p is None) == (q is None)
            if p is not None:
                assert torch.equal(p, q) and p.stride() == q.stride() and p.dtype == q.dtype and not p.requires_grad and not q.requires_grad, n
    gf.last_device_status()


@pytest.mark.gpu
def test_other_forms_are_what_python_makes_of_them(both):
    m = make()
    x, w, x2, w2, ws, dy, head, t = (m[n] for n in ("x", "w", "x2", "w2", "ws", "dy", "head", "t"))
    lse = gf.vocab_loss(x, head, t)[1]
    refused = [lambda: gf.gated_linear(x, w, x, w2), lambda: gf.gated_linear(x, w, None, w2), lambda: gf.gated_linear(x, w, x2), lambda: gf.gated_linear(x.float(), w),
               lambda: gf.gated_linear(x, w.t()), lambda: gf.gated_linear(x, w.cpu()), lambda: gf.gated_linear(x[..., ::2], w[::2]), lambda: gf.gated_linear(x, w, act="none"),
               lambda: gf.gated_linear(x, w[:, :100].contiguous()), lambda: gf.gated_linear_backward(x, w, dy[:1]), lambda: gf.gated_linear_backward(x, w, dy.float()),
               lambda: gf.gated_linear_backward(x, w, dy, x2, ws), lambda: gf.vocab_loss(x, head, t.int()), lambda: gf.vocab_loss(x, head, t[:1]),
               lambda: gf.vocab_loss(x, head[:0], t), lambda: gf.vocab_loss(x[..., :60].contiguous(), head[:, :60].contiguous(), t),
               lambda: gf.vocab_loss_backward(x, head, t, lse.double()), lambda: gf.vocab_loss_backward(x, head, t, lse, m["d"][:1]),
               lambda: gf.layernorm_heads_backward(m["y"], m["dout"].float()), lambda: gf.layernorm_heads_backward(m["y"], m["dout"][:1]),
               lambda: gf.layernorm_heads_backward(m["y"], m["dout"], m["gamma"][:100]), lambda: gf.layernorm_heads_backward(m["y"], m["dout"], m["gamma"], -1.0)]
    for n, call in enumerate(refused):
        a, b = both(call)
        assert isinstance(a, tuple) and isinstance(a[0], type) and a == b, (n, a, b)
