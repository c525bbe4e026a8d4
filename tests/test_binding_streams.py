"""Where the binding allocates and copies: a call with stream= makes its outputs, its workspace and its copies on the stream that it launches on, so that the
caching allocator hands none of that memory on before the kernels have run, and what it hands over lives until the call.

Without a GPU the Python code is watched: CPU tensors pose as CUDA ones, streams are stand-ins, the library notes what it is called with."""
import contextlib
import ctypes

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

import paper_2407_12077_b200 as gf

BF, F32 = torch.bfloat16, torch.float32
CURRENT, SIDE = 7, 99                                # raw handles


class Side:
    cuda_stream = SIDE

    def __init__(self, handle=SIDE, device=None):
        self.cuda_stream, self.device, self.device_index = handle, torch.device("cuda", 0), 0


class Watch(TorchDispatchMode):
    """Notes the stream under which each operation that makes memory runs."""

    def __init__(self, host):
        super().__init__()
        self.host = host

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if any(n in func.__name__ for n in ("empty", "clone", "copy", "zeros", "new_", "contiguous")):
            self.host.made.append((func.__name__, self.host.stream))
        return out


class Host:
    """The library, the device and its streams as the binding sees them."""

    def __init__(self):
        self.stream, self.made, self.calls, self.look, self.recorded = CURRENT, [], [], None, []

    def __getattr__(self, name):
        if not name.startswith("gf_"):
            raise AttributeError(name)

        def call(*args):
            if name.endswith("bytes"):
                return 4096
            if name.startswith("gf_wkv6_set") or name == "gf_wkv6_launch_count":
                return 0
            self.calls.append((name, args[-1], self.stream))
            if self.look:
                self.look(args)
            return 0

        return call


@pytest.fixture
def host(monkeypatch):
    h = Host()
    monkeypatch.setattr(gf, "_lib", h)
    monkeypatch.setattr(gf, "_native", None)
    monkeypatch.setattr(gf, "_workspace", None)
    gf._workspace_need.cache_clear()
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: h.recorded.append((self.data_ptr(), s.cuda_stream)), raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "Stream", Side)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Side)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Side(h.stream))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: h.stream, raising=False)

    @contextlib.contextmanager
    def under(s):
        before, h.stream = h.stream, s.cuda_stream
        try:
            yield
        finally:
            h.stream = before

    monkeypatch.setattr(torch.cuda, "stream", under)
    yield h
    gf._workspace_need.cache_clear()


def tensors():
    z = torch.zeros
    d = z(1, 8, 2, 64, dtype=BF)
    p = z(8, 2, 64, dtype=BF)
    s = z(2, 2, 64, dtype=BF)
    return dict(d=d, f=d.float(), p=p, pf=p.float(), s=s, u=z(2, 64), cu=torch.tensor([0, 8], dtype=torch.int32), st=z(2, 2, 64, 64), ws=z(1 << 13, dtype=torch.uint8), x=z(8, 64, dtype=BF),
                w=z(64, 72, dtype=BF), x2=z(8, 80, dtype=BF), w2=z(80, 72, dtype=BF), dy=z(8, 72, dtype=BF), head=z(100, 64, dtype=BF), t=z(8, dtype=torch.int64), lse=z(8),
                lam=z(64), A=z(64, 16, dtype=BF), B=z(16, 64, dtype=BF), x3=z(1, 8, 64, dtype=BF))


def run_all():
    """name -> call(stream) of every function that takes one and allocates."""
    m = tensors()
    d, f, p, pf, s, u, cu, st, ws, x, w, x2, w2, dy, head, t, lse = (m[n] for n in ("d", "f", "p", "pf", "s", "u", "cu", "st", "ws", "x", "w", "x2", "w2", "dy", "head", "t", "lse"))
    wide = torch.zeros(2, 128)                       # a gamma that has to be copied
    return {
        "prefill": lambda q: gf.prefill(d, d, d, d, u, stream=q),
        "prefill f32": lambda q: gf.prefill(f, f, f, f, u, stream=q),
        "prefill_c2": lambda q: gf.prefill_c2(d, d, d, d, stream=q),
        "prefill_varlen": lambda q: gf.prefill_varlen(p, p, p, p, u, cu, 8, stream=q),
        "prefill_varlen f32": lambda q: gf.prefill_varlen(pf, pf, pf, pf, u, cu, 8, stream=q),
        "prefill_varlen_c2": lambda q: gf.prefill_varlen_c2(p, p, p, p, None, cu, 8, stream=q),
        "prefill_train": lambda q: gf.prefill_train(d, d, d, d, u, ws, stream=q),
        "prefill_varlen_train": lambda q: gf.prefill_varlen_train(p, p, p, p, u, cu, 8, ws, stream=q),
        "step": lambda q: gf.step(s, s, s, s, u, None, stream=q),
        "step_c2": lambda q: gf.step_c2(s, s, s, s, None, None, stream=q),
        "bind_step": lambda q: gf.bind_step(s, s, s, s, u, st, stream=q)[0](),
        "backward": lambda q: gf.backward(d, d, d, d, u, d, stream=q),
        "backward f32": lambda q: gf.backward(f, f, f, f, u, f, stream=q),
        "backward_c2": lambda q: gf.backward_c2(d, d, d, d, d, stream=q),
        "backward_varlen": lambda q: gf.backward_varlen(p, p, p, p, u, p, cu, 8, stream=q),
        "sequence_summary": lambda q: gf.sequence_summary(d, d, d, stream=q),
        "fold_summaries": lambda q: gf.fold_summaries(None, torch.zeros(1, 1, 2, gf.SUMMARY_FLOATS), 1, stream=q),
        "layernorm_heads": lambda q: gf.layernorm_heads(d, wide[:, :64], wide[:, :64], stream=q),
        "layernorm_heads_backward": lambda q: gf.layernorm_heads_backward(d, d, wide[:, :64], stream=q),
        "key_compress": lambda q: gf.key_compress(x, w, stream=q),
        "gated_linear": lambda q: gf.gated_linear(x, w, x2, w2, stream=q),
        "gated_linear_backward": lambda q: gf.gated_linear_backward(x, w, dy, x2, w2, stream=q),
        "vocab_loss": lambda q: gf.vocab_loss(x, head, t, stream=q),
        "vocab_loss_backward": lambda q: gf.vocab_loss_backward(x, head, t, lse, stream=q),
        "decay_logit": lambda q: gf.decay_logit(m["x3"], m["lam"], m["A"], m["B"], m["lam"], m["A"], m["B"], m["lam"], stream=q),
    }


NAMES = list(run_all())


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("how", ["stream", "handle"])
def test_memory_is_made_on_the_stream_of_the_launch(host, name, how):
    call = run_all()[name]
    with Watch(host):
        call(Side() if how == "stream" else SIDE)
    made = [m for m in host.made if name != "fold_summaries" or "zeros" not in m[0]]      # (its own argument above)
    assert made and all(stream == SIDE for _, stream in made), made
    assert host.calls and all(handle == SIDE for _, handle, _ in host.calls)
    assert host.stream == CURRENT


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("stream", [None, CURRENT])
def test_without_another_stream_nothing_is_entered(host, name, stream, monkeypatch):
    def entered(s):
        raise AssertionError("a stream context for the stream that is current already")

    monkeypatch.setattr(torch.cuda, "stream", entered)
    run_all()[name](stream)
    assert host.calls and all(handle == CURRENT for _, handle, _ in host.calls)


def test_a_stream_of_another_device_is_refused(host):
    there = Side()
    there.device, there.device_index = torch.device("cuda", 1), 1
    for name, call in run_all().items():
        with pytest.raises(ValueError, match="device"):
            call(there)
    assert not host.calls and host.stream == CURRENT


def test_scratch_is_noted_on_every_stream_that_uses_it(host):
    """The registered scratch outlives calls on several streams: torch's allocator is told of each before the scratch can be dropped."""
    d, u = torch.zeros(1, 8, 2, 64, dtype=BF), torch.zeros(2, 64)
    gf.prefill(d, d, d, d, u)
    first = gf._workspace.data_ptr()
    gf.prefill(d, d, d, d, u, stream=Side())
    gf.prefill_c2(d, d, d, d, stream=SIDE)
    gf.prefill(d, d, d, d, u)
    assert host.recorded == [(first, CURRENT), (first, SIDE)]
    mine = torch.zeros(1 << 13, dtype=torch.uint8)
    gf.set_workspace(mine)                           # a buffer of the caller's, wherever it was made
    gf.prefill(d, d, d, d, u, stream=SIDE)
    assert host.recorded[2:] == [(mine.data_ptr(), SIDE)]
    gf.set_workspace(None)
    gf.prefill(d, d, d, d, u, stream=SIDE)
    assert len(host.recorded) == 4 and host.recorded[3][1] == SIDE
    gf.prefill(d.float(), d.float(), d.float(), d.float(), u, stream=Side(55))      # (no scratch in fp32)
    assert len(host.recorded) == 4


@pytest.fixture
def default_stream(host, monkeypatch):
    """torch.cuda.ExternalStream(0) is a stream from torch's pool; handle 0 is the default stream."""
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Side(handle or 1000))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: Side(0))


@pytest.mark.parametrize("name", NAMES)
def test_handle_zero_is_the_default_stream(host, default_stream, name):
    call = run_all()[name]
    with Watch(host):
        call(0)
    made = [m for m in host.made if name != "fold_summaries" or "zeros" not in m[0]]
    assert made and all(stream == 0 for _, stream in made), made
    assert host.calls and all(handle == 0 for _, handle, _ in host.calls)


def test_scratch_is_noted_on_the_default_stream(host, default_stream):
    d, u = torch.zeros(1, 8, 2, 64, dtype=BF), torch.zeros(2, 64)
    gf.set_workspace(torch.zeros(1 << 13, dtype=torch.uint8))
    gf.prefill(d, d, d, d, u, stream=0)
    host.stream = 0                                  # (the current one from here on)
    gf.prefill(d, d, d, d, u)
    assert [handle for _, handle in host.recorded] == [0]
