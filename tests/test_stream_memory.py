"""Where the Python calls take memory from when they are given a stream: from that stream's pool, so that a block is never one that another
stream has given back with work still queued on it.  The library and the streams are stand-ins here (no GPU)."""
import pytest
import torch

from paper_2603_06588_amd import binding


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream, self.device = handle, device


CURRENT = Stream(5)


class Streams:
    """The current stream's name, as torch.cuda.stream() switches it."""

    def __init__(self):
        self.current, self.taken, self.recorded = CURRENT, [], []

    def switch(self, stream):
        outer = self

        class Context:
            def __enter__(self):
                self.before, outer.current = outer.current, stream

            def __exit__(self, *_):
                outer.current = self.before
        return Context()


class Library:
    """Accepts every call; any scratch is 512 bytes."""

    def __getattr__(self, name):
        return (lambda *a: 512) if name.endswith("_workspace_bytes") else (lambda *a: 0)


@pytest.fixture
def streams(monkeypatch):
    s = Streams()

    def on_host(make):
        def made(*args, **kw):
            kw.pop("device", None)
            t = make(*args, **kw)
            s.taken.append((s.current, t))
            return t
        return made
    monkeypatch.setattr(binding.torch, "empty", on_host(torch.empty))
    monkeypatch.setattr(binding.torch, "empty_like", on_host(torch.empty_like))
    monkeypatch.setattr(torch.cuda, "stream", s.switch)
    monkeypatch.setattr(torch.cuda, "Stream", Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: s.current)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: s.recorded.append((stream, t)))
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "pages_workspace_bytes", lambda *a: 512)
    monkeypatch.setattr(binding, "_look", lambda where, like, spec, *tensors: (0,) + (0, ()) * len(tensors))
    return s


def calls():
    f, i = torch.zeros, lambda *n: torch.zeros(n, dtype=torch.int32)
    q, cache = f(3, 2, 64), f(4, 1, 16, 64)
    pages = binding.HookPagesArgs(1, 2, 4, 16)
    return {
        "hook_attn_probe": (lambda s: binding.hook_attn_probe(q, cache, cache, i(1, 2), i(1), i(2), probe_heads=i(1), stream=s), 2, 3),
        "hook_span_mass": (lambda s: (binding.hook_span_mass(q, cache, i(1, 2), i(1), i(2), i(1), 1, i(1, 1), 2, i(1, 2, 2), stream=s),), 1, 2),
        "hook_capture_qk": (lambda s: binding.hook_capture_qk(q, cache, i(1, 2), i(1), i(2), i(1), 1, i(1, 1), i(1), i(2), 5, stream=s), 2, 2),
        "hook_reduce_mass": (lambda s: (binding.hook_reduce_mass(f(1, 2, 3, 4), 0, stream=s),), 1, 1),
        "hook_pages_append, hook_pages_compact": (lambda s: binding._pages_data("pages", pages, [], i(1, 2), None, 0, s) and (), 0, 1),
    }


class Handle:
    cuda_stream = 77


@pytest.mark.parametrize("name", list(calls()))
@pytest.mark.parametrize("known", [True, False])      # a torch stream, and an object that has its handle alone
def test_memory_comes_from_the_stream_of_the_call(name, known, streams, monkeypatch):
    call, results, allocations = calls()[name]
    stream = Stream(77) if known else Handle()
    monkeypatch.setattr(binding, "_stream_handle", lambda s: 77)
    out = call(stream)
    assert len(streams.taken) == allocations and all(on.cuda_stream == 77 for on, _ in streams.taken)
    # a stream known by its handle alone belongs to the GPU of the call's tensors
    assert known or all(on.device in (0, torch.device("cpu")) for on, _ in streams.taken)
    # results outlive the call and are read on the current stream, scratch is not
    assert len(out) == results and {id(t) for t in out} == {id(t) for _, t in streams.recorded}
    assert all(on is CURRENT for on, _ in streams.recorded)


@pytest.mark.parametrize("name", list(calls()))
@pytest.mark.parametrize("given", [False, True])
def test_calls_on_the_current_stream_record_nothing(name, given, streams, monkeypatch):
    call, _, allocations = calls()[name]
    monkeypatch.setattr(binding, "_stream_handle", lambda s: 5)
    call(CURRENT if given else None)
    assert len(streams.taken) == allocations and all(on is CURRENT for on, _ in streams.taken) and not streams.recorded
