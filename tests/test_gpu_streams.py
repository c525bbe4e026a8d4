"""Calls with stream=: their memory is theirs until their kernels have run, whatever the current stream allocates meanwhile."""
import pytest
import torch

import paper_2407_12077_b200 as gf
from paper_2407_12077_b200 import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def make(seed):
    g = torch.Generator().manual_seed(seed)

    def r(*s, std=1.0, dtype=BF):
        return (torch.randn(*s, generator=g) * std).to(dtype).to(DEV)

    rows, D, F, V = 700, 256, 520, 3001
    d = synth.make_dense(2, 300, 4, 64, "bf16", seed=seed, device=DEV, state_std=0.1)
    return dict(y=r(rows, 4, 64), dout=r(rows, 4, 64), wide=r(4, 128, dtype=torch.float32), wide2=r(4, 128, dtype=torch.float32), x=r(rows, D), w=r(D, F, std=D ** -0.5), x2=r(rows, 328),
                w2=r(328, F, std=328 ** -0.5), dy=r(rows, F), head=r(V, D, std=2 * D ** -0.5), t=torch.randint(0, V, (rows,), generator=g).to(DEV), d=d, dyr=r(2, 300, 4, 64))


def calls(m):
    """name -> call(stream) -> outputs"""
    gamma, beta, d = m["wide"][:, :64], m["wide2"][:, :64], m["d"]
    lse = gf.vocab_loss(m["x"], m["head"], m["t"])[1]
    torch.cuda.synchronize()
    return {
        "layernorm_heads": lambda q: (gf.layernorm_heads(m["y"], gamma, beta, stream=q),),
        "layernorm_heads_backward": lambda q: gf.layernorm_heads_backward(m["y"], m["dout"], gamma, stream=q),
        "gated_linear": lambda q: (gf.gated_linear(m["x"], m["w"], m["x2"], m["w2"], stream=q),),
        "gated_linear_backward": lambda q: gf.gated_linear_backward(m["x"], m["w"], m["dy"], m["x2"], m["w2"], stream=q),
        "vocab_loss": lambda q: gf.vocab_loss(m["x"], m["head"], m["t"], stream=q),
        "vocab_loss_backward": lambda q: gf.vocab_loss_backward(m["x"], m["head"], m["t"], lse, stream=q),
        "prefill": lambda q: gf.prefill(d.r, d.k, d.v, d.x, d.u, d.state_in, stream=q),
        "backward": lambda q: gf.backward(d.r, d.k, d.v, d.x, d.u, m["dyr"], d.state_in, stream=q),
        "backward_c2": lambda q: gf.backward_c2(d.r, d.k, d.v, d.x, m["dyr"], d.state_in, stream=q),
    }


NAMES = ["layernorm_heads", "layernorm_heads_backward", "gated_linear", "gated_linear_backward", "vocab_loss", "vocab_loss_backward", "prefill", "backward", "backward_c2"]
# blocks of every size that the calls above may have given back, and then some
SIZES = [512 << i for i in range(17)] + [n << s for n in (1, 3, 5, 7) for s in (20, 22)]


def scribble():
    """What the current stream is given next, filled with bytes that make NaNs."""
    return [torch.full((n,), 255, dtype=torch.uint8, device=DEV) for n in SIZES for _ in range(2)]


def equal(a, b, what):
    for p, q in zip(a, b, strict=True):
        assert (p is None) == (q is None) and (p is None or torch.equal(p, q)), what


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("handle", [False, True])
def test_current_stream_is_given_none_of_a_calls_memory(name, handle):
    call = calls(make(1))[name]
    want = call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(4_000_000)             # (the call's kernels wait behind this for about 2 ms)
        got = call(side.cuda_stream if handle else side)
        held = scribble()
        torch.cuda.synchronize()
        gf.last_device_status(side)
        equal(got, want, name)
        del held, got


def test_two_streams_at_a_time():
    runs = [calls(make(s)) for s in (1, 2)]
    want = [{n: c(None) for n, c in r.items() if n != "prefill"} for r in runs]      # (a prefill's registered scratch is for one stream at a time)
    sides = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [{}, {}]
        for n in want[0]:
            for i, r in enumerate(runs):
                got[i][n] = r[n](sides[i])
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for n in w:
                equal(g[n], w[n], n)
    gf.last_device_status()


@pytest.mark.parametrize("how", ["stream=", "context"])
def test_dropped_scratch_is_not_handed_on_while_another_stream_uses_it(how):
    """A prefill that splits: scratch made on the current stream, used on another one, replaced and dropped while that one still runs."""
    d = synth.make_dense(1, 4096, 4, 64, "bf16", seed=3, device=DEV, state_std=0.1)
    need = gf.workspace_bytes(1, 4096, 4)
    assert need > 0
    gf.set_workspace(None)
    want = gf.prefill(d.r, d.k, d.v, d.x, d.u, d.state_in)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        gf.set_workspace(torch.empty(need, dtype=torch.uint8, device=DEV))
        with torch.cuda.stream(side):
            torch.cuda._sleep(4_000_000)
            got = gf.prefill(d.r, d.k, d.v, d.x, d.u, d.state_in) if how == "context" else None
        if got is None:
            got = gf.prefill(d.r, d.k, d.v, d.x, d.u, d.state_in, stream=side)
        gf.set_workspace(None)
        held = [torch.full((need,), 255, dtype=torch.uint8, device=DEV) for _ in range(3)]
        torch.cuda.synchronize()
        gf.last_device_status(side)
        equal(got, want, how)
        del held


@pytest.mark.parametrize("name", NAMES)
def test_default_stream_by_its_handle_while_another_one_is_current(name):
    call = calls(make(2))[name]
    want = call(None)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(4_000_000)
        with torch.cuda.stream(side):
            got = call(0)
            held = scribble()
        torch.cuda.synchronize()
        gf.last_device_status()
        equal(got, want, name)
        del held, got
