"""Refusals of the operators around the recurrence (gradient of the norm, gated linear block, vocabulary loss): bad arguments are
turned away before anything touches CUDA, at the C interface and in the binding."""
import ctypes

import pytest
import torch

import paper_2407_12077_b200 as gf

A = 0x1000                                       # fake 16-byte aligned "device pointers", never dereferenced
P = [A + 0x100 * i for i in range(12)]
BIG = 1 << 60
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 4
F = ctypes.c_float


def call(name, *args):
    return getattr(gf.load_library(), name)(*args)


def changed(args, **at):
    args = list(args)
    for k, v in at.items():
        args[int(k[1:])] = v
    return args


@pytest.mark.parametrize("name", ["gf_c2_layernorm_backward", "gf_c2_layernorm_backward_f32"])
def test_norm_gradient(name):
    #       y     gamma eps       dout  dy    dgamma dbeta rows H   N   ws    bytes stream
    good = [P[0], P[1], F(1e-5), P[2], P[3], P[4], P[5], 4, 32, 64, P[6], BIG, None]
    for i in (0, 3, 4):
        assert call(name, *changed(good, **{f"_{i}": None})) == INVALID
    for i in (0, 1, 3, 4, 5, 6, 10):
        assert call(name, *changed(good, **{f"_{i}": A + 4})) == INVALID
    assert call(name, *changed(good, _7=-1)) == INVALID
    assert call(name, *changed(good, _2=F(-1.0))) == INVALID and call(name, *changed(good, _2=F(float("nan")))) == INVALID
    assert call(name, *changed(good, _8=3, _9=5)) == UNSUPPORTED and call(name, *changed(good, _8=129)) == UNSUPPORTED
    assert call(name, *changed(good, _8=0)) == OK                       # no channels
    assert call(name, *changed(good, _5=None, _6=None, _7=0)) == OK     # no rows, no sums wanted
    assert call("gf_c2_layernorm_backward_workspace_bytes", 3, 5) == 0


def test_gated_linear():
    #       x     w     x2    w2    act y     rows K1  K2  F  stream
    good = [P[0], P[1], P[2], P[3], 0, P[4], 8, 64, 128, 64, None]
    name = "gf_gated_linear"
    for i in (0, 1, 5):
        assert call(name, *changed(good, **{f"_{i}": None})) == INVALID
    for i in (0, 1, 2, 3, 5):
        assert call(name, *changed(good, **{f"_{i}": A + 2})) == INVALID
    for i in (0, 1, 2, 3):
        assert call(name, *changed(good, _5=P[i])) == INVALID            # y is an input
    for act in (-1, 4):
        assert call(name, *changed(good, _4=act)) == INVALID
    for i in (6, 7, 8, 9):
        assert call(name, *changed(good, **{f"_{i}": -8})) == INVALID
    assert call(name, *changed(good, _2=None)) == INVALID                # x2 = x with another depth
    assert call(name, *changed(good, _3=None)) == INVALID                # x2 without w2
    assert call(name, *changed(good, _2=None, _3=None)) == INVALID       # a depth without w2
    for i, v in ((7, 0), (8, 0), (7, 60), (8, 4), (9, 100)):
        assert call(name, *changed(good, **{f"_{i}": v})) == UNSUPPORTED
    assert call(name, *changed(good, _6=(1 << 31))) == UNSUPPORTED
    assert call(name, *changed(good, _6=0)) == OK and call(name, *changed(good, _9=0)) == OK


def test_gated_linear_backward():
    #       x     w     x2    w2    act dy    dx    dw    dx2   dw2   rows K1 K2   F   ws     bytes stream
    good = [P[0], P[1], P[2], P[3], 0, P[4], P[5], P[6], P[7], P[8], 8, 64, 128, 64, P[9], BIG, None]
    name = "gf_gated_linear_backward"
    for i in (0, 1, 5, 6, 7, 8, 9):
        assert call(name, *changed(good, **{f"_{i}": None})) == INVALID
    for i in (0, 1, 2, 3, 5, 6, 7, 8, 9, 14):
        assert call(name, *changed(good, **{f"_{i}": A + 8})) == INVALID
    for out in (6, 7, 8, 9):
        for other in (0, 1, 2, 3, 5, 6, 7, 8, 9):
            if out != other:
                assert call(name, *changed(good, **{f"_{out}": good[other]})) == INVALID
    one = changed(good, _2=None, _3=None, _8=None, _9=None, _12=0)       # no second product
    assert call(name, *changed(one, _9=P[8])) == INVALID and call(name, *changed(one, _8=P[7])) == INVALID
    same = changed(good, _2=None, _8=None, _12=64)                       # x2 = x
    assert call(name, *changed(same, _8=P[7])) == INVALID and call(name, *changed(same, _12=128)) == INVALID
    for args, K2, is_same in ((good, 128, 0), (one, 0, 0), (same, 64, 1)):
        need = call("gf_gated_linear_backward_workspace_bytes", 8, 64, K2, 64, is_same)
        assert need >= 8 * 64 * 2 * (2 if K2 else 1)
        assert call(name, *changed(args, _15=need - 1)) == WORKSPACE and call(name, *changed(args, _14=None)) == WORKSPACE
    assert call(name, *changed(good, _11=60)) == UNSUPPORTED
    assert call("gf_gated_linear_backward_workspace_bytes", 0, 64, 64, 64, 1) == 0
    assert call(name, *changed(good, _6=None, _7=None, _8=None, _9=None, _10=0)) == OK      # no rows, nothing to write


def test_vocab_loss():
    #       x     w     t     loss  lse   rows D  V    ws    bytes stream
    good = [P[0], P[1], P[2], P[3], P[4], 8, 64, 100, P[5], BIG, None]
    name = "gf_vocab_loss"
    for i in (0, 1, 2, 3, 4):
        assert call(name, *changed(good, **{f"_{i}": None})) == INVALID
    for i in (0, 1, 8):
        assert call(name, *changed(good, **{f"_{i}": A + 8})) == INVALID
    assert call(name, *changed(good, _2=A + 4)) == INVALID and call(name, *changed(good, _3=A + 2)) == INVALID and call(name, *changed(good, _4=A + 2)) == INVALID
    assert call(name, *changed(good, _4=P[3])) == INVALID
    for i, v in ((5, -1), (6, -8), (7, 0), (7, -1)):
        assert call(name, *changed(good, **{f"_{i}": v})) == INVALID
    for i, v in ((6, 0), (6, 60), (5, 1 << 31), (7, 1 << 31)):
        assert call(name, *changed(good, **{f"_{i}": v})) == UNSUPPORTED
    assert call(name, *changed(good, _5=(1 << 31) - 300, _7=(1 << 31) - 300)) == UNSUPPORTED      # more tiles than a launch counts
    need = call("gf_vocab_loss_workspace_bytes", 8, 100)
    assert call(name, *changed(good, _9=need - 1)) == WORKSPACE and call(name, *changed(good, _8=None)) == WORKSPACE
    assert call(name, *changed(good, _5=0)) == OK


def test_vocab_loss_backward():
    #       x     w     t     lse   dloss dx    dw    rows D  V    ws    bytes stream
    good = [P[0], P[1], P[2], P[3], P[4], P[5], P[6], 8, 64, 100, P[7], BIG, None]
    name = "gf_vocab_loss_backward"
    for i in (0, 1, 2, 3, 5, 6):
        assert call(name, *changed(good, **{f"_{i}": None})) == INVALID
    for i in (0, 1, 2, 5, 6, 10):
        assert call(name, *changed(good, **{f"_{i}": A + 4})) == INVALID
    assert call(name, *changed(good, _3=A + 2)) == INVALID and call(name, *changed(good, _4=A + 2)) == INVALID
    for out, other in ((5, 0), (5, 1), (6, 0), (6, 1), (6, 5)):
        assert call(name, *changed(good, **{f"_{out}": good[other]})) == INVALID
    need = call("gf_vocab_loss_backward_workspace_bytes", 8, 64, 100)
    assert call(name, *changed(good, _11=need - 1)) == WORKSPACE and call(name, *changed(good, _10=None)) == WORKSPACE
    assert call(name, *changed(good, _8=4)) == UNSUPPORTED and call(name, *changed(good, _9=0)) == INVALID
    assert call(name, *changed(good, _6=None, _7=0)) == OK
    # the workspace holds one piece of the vocabulary: bounded in V, and in the number of rows up to 2 KB for each
    sizes = [call("gf_vocab_loss_backward_workspace_bytes", 8192, 64, v) for v in (1 << 16, 1 << 20, 1 << 24)]
    assert max(sizes) <= (512 << 20) + 8192 * 64 * 4


def test_binding_refuses():
    bf = torch.bfloat16
    x, w, t = torch.zeros(4, 64, dtype=bf), torch.zeros(64, 64, dtype=bf), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        gf.gated_linear(x, w)
    with pytest.raises(ValueError, match="CUDA"):
        gf.gated_linear_backward(x, w, x)
    with pytest.raises(ValueError, match="CUDA"):
        gf.vocab_loss(x, w, t)
    with pytest.raises(ValueError, match="CUDA"):
        gf.vocab_loss_backward(x, w, t, torch.zeros(4))
    with pytest.raises(ValueError, match="CUDA"):
        gf.layernorm_heads_backward(torch.zeros(4, 1, 64), torch.zeros(4, 1, 64), want_params=False)
    with pytest.raises(ValueError, match="act must be"):
        gf.gated_linear(x, w, act="tanh")
    with pytest.raises(ValueError, match="x2 without w2"):
        gf.gated_linear(x, w, x2=x)
    with pytest.raises(TypeError):
        gf.layernorm_heads_backward(torch.zeros(4, 1, 64, dtype=torch.float16), torch.zeros(4, 1, 64, dtype=torch.float16))
