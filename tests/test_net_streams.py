"""Which stream's memory a call of the network's operators on another stream works in: a block that the caching allocator hands out is free only in the
order of the stream that it is asked for on.  On the CPU, with the library and the allocator stood in for."""
import contextlib

import pytest
import torch

from paper_2503_10017_amd import net


class OnDevice(torch.Tensor):
    """A CPU tensor that says it is on the device, and notes whom it is recorded for."""
    is_cuda = property(lambda self: True)

    def record_stream(self, stream):
        self.recorded = getattr(self, "recorded", []) + [stream]


class Library:
    """Every function: 1024 bytes of workspace, or status 0."""

    def __getattr__(self, name):
        return lambda *args: 1024 if name.endswith("workspace_bytes") else 0


class Stream:
    cuda_stream = 0x77


class Allocator:
    def __init__(self):
        self.current, self.taken = "usual", []

    def give(self, of):
        def make(*args, **kw):
            t = of(*args, **kw).as_subclass(OnDevice)
            self.taken.append((self.current, t))
            return t
        return make

    @contextlib.contextmanager
    def stream(self, s):
        before = self.current
        self.current = before if s is None else s
        yield
        self.current = before


@pytest.fixture
def allocator(monkeypatch):
    a = Allocator()
    monkeypatch.setattr(net, "load_library", Library)
    monkeypatch.setattr(torch, "empty", a.give(torch.empty))
    monkeypatch.setattr(torch, "empty_like", a.give(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "stream", a.stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: a.current)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    return a


def given(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


X, W, V = given(8, 64), given(32, 64), given(64)
STATS = given(8, dtype=torch.float32)
Q, K, LSE = given(8, 4, 64), given(9, 2, 64), given(8, 4, dtype=torch.float32)
CALLS = {
    "fnn_layer_norm": lambda **kw: net.fnn_layer_norm(X, V, V, want_stats=True, **kw),
    "fnn_layer_norm_backward": lambda **kw: net.fnn_layer_norm_backward(X, X, STATS, STATS, V, **kw),
    "fnn_linear": lambda **kw: net.fnn_linear(X, W, want_pre=True, **kw),
    "fnn_linear_backward": lambda **kw: net.fnn_linear_backward(given(8, 32), X, W, **kw),
    "fnn_attention": lambda **kw: net.fnn_attention(Q, K, K, **kw),
    "fnn_attention_backward": lambda **kw: net.fnn_attention_backward(Q, Q, K, K, Q, LSE, **kw),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_on_another_stream_takes_its_memory_there(allocator, name):
    side = Stream()
    results = [t for t in CALLS[name](stream=side) if t is not None]
    assert results and len(allocator.taken) == len(results) + (name != "fnn_layer_norm")     # and a workspace
    assert all(of is side for of, _ in allocator.taken)
    # what is returned is read by the caller on the current stream, and may be dropped before that has happened
    assert all("usual" in getattr(t, "recorded", []) for t in results)
    assert allocator.current == "usual"


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_on_the_current_stream_takes_its_memory_there(allocator, name):
    results = [t for t in CALLS[name]() if t is not None]
    assert results and all(of == "usual" for of, _ in allocator.taken)
    assert not any(hasattr(t, "recorded") for _, t in allocator.taken)
