"""Which stream's memory a matching call on another stream works in (as tests/test_net_streams.py, for the functions of fnn.h)."""
import pytest
import torch

from paper_2503_10017_amd import binding
from test_net_streams import Allocator, Library, Stream, given


class Matching(Library):
    """The same, and the workspace sizes of fnn.h."""

    def __getattr__(self, name):
        return lambda *args: 4096 if "workspace_bytes" in name else 0


@pytest.fixture
def allocator(monkeypatch):
    a = Allocator()
    monkeypatch.setattr(binding, "load_library", Matching)
    monkeypatch.setattr(torch, "empty", a.give(torch.empty))
    monkeypatch.setattr(torch.cuda, "stream", a.stream)

    class Current(str):
        cuda_stream = 0

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Current(a.current))
    return a


MAP, OTHER = given(100, 24), given(90, 24)
SEEDS = given(1, 10, dtype=torch.int32)
PAIRS, COUNT = given(1, 10, 2, dtype=torch.int32), given(1, dtype=torch.int32)
CALLS = {
    "fnn_nearest": lambda **kw: binding.fnn_nearest(MAP, OTHER, compute="bf16", **kw),
    "fnn_reciprocal": lambda **kw: binding.fnn_reciprocal(MAP, OTHER, SEEDS, compute="bf16", **kw),
    "fnn_mutual_dense": lambda **kw: binding.fnn_mutual_dense(MAP, OTHER, compute="bf16", **kw),
    "fnn_nearest_blocked": lambda **kw: binding.fnn_nearest_blocked(MAP, OTHER, 32, compute="bf16", **kw),
    "fnn_pairs_to_pixels": lambda **kw: binding.fnn_pairs_to_pixels(PAIRS, COUNT, 100, 10, 90, 10, **kw),
}


def outputs(result):
    return list(result.values()) if isinstance(result, dict) else list(result)


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_on_another_stream_takes_its_memory_there(allocator, name):
    side = Stream()
    results = outputs(CALLS[name](stream=side))
    assert results and len(allocator.taken) == len(results) + (name != "fnn_pairs_to_pixels")     # and a workspace
    assert all(of is side for of, _ in allocator.taken)
    assert all("usual" in getattr(t, "recorded", []) for t in results)
    assert allocator.current == "usual"


@pytest.mark.parametrize("name", list(CALLS))
def test_a_call_on_the_current_stream_takes_its_memory_there(allocator, name):
    results = outputs(CALLS[name]())
    assert results and all(of == "usual" for of, _ in allocator.taken)
    assert not any(hasattr(t, "recorded") for _, t in allocator.taken)
