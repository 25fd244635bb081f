"""Which stream an operator's call runs on (paper_2601_01473_gb300/ops.py)."""
import collections
import contextlib

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2601_01473_gb300 import Graph, ops


class _Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream, self.device = handle, device


def test_a_stream_is_one_of_the_arguments_device(monkeypatch):
    """Without a GPU: a handle becomes a stream of the tensors' device whatever device is
    current, and a stream of another device is refused."""
    ran_on, kept_for = [], []
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", _Stream)
    monkeypatch.setattr(torch.cuda, "stream", lambda s: ran_on.append(s) or contextlib.nullcontext())
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: kept_for.append(s))
    with FakeTensorMode():
        tensors = [torch.empty(3, device=f"cuda:{i}") for i in range(2)]
    for t in tensors:
        for stream in (77, _Stream(77, t.device)):
            assert ops._on_stream(stream, lambda *args: args, 1.5, t, None) == (1.5, t, None)
            assert ran_on[-1].cuda_stream == 77 and ran_on[-1].device == t.device
            assert kept_for[-1] is ran_on[-1]
    with pytest.raises(ValueError, match="cuda:1.*cuda:0"):
        ops._on_stream(_Stream(5, tensors[1].device), lambda *args: args, tensors[0])


def test_arguments_off_the_gpu_are_refused_with_a_stream_too():
    with pytest.raises(ValueError, match="CUDA device"):
        ops.embedding_lookup(torch.zeros(4, 8), torch.zeros(3, dtype=torch.int32), stream=0)
    with pytest.raises(TypeError, match="2-D"):
        ops.mx4_quantize(None, stream=0)


@pytest.mark.gpu
def test_a_call_is_ordered_by_the_stream_that_is_named(cuda_device):
    """By its object and by its handle: what a stream has before the call is there for it, and
    what it has after sees its results."""
    for named in (lambda s: s, lambda s: s.cuda_stream):
        stream = torch.cuda.Stream()
        table = torch.zeros(4_000_000, 64, device=cuda_device)
        ids = torch.full((100_000,), 3_999_999, dtype=torch.int32, device=cuda_device)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            for v in range(1, 9):
                table.fill_(v)
        got = ops.embedding_lookup(table, ids, stream=named(stream))
        with torch.cuda.stream(stream):
            table.fill_(-1)
            total = got.sum()
        torch.cuda.synchronize()
        assert float(total) == 8 * 64 * 100_000
    ops.check()


def test_no_handle_is_the_default_stream(monkeypatch):
    """Without a GPU: torch makes a stream of its own of an ExternalStream without a handle."""
    device = torch.device("cuda", 1)
    default = _Stream(0, device)
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", _Stream)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda d: default if d == device else None)
    assert ops._stream_of(0, device) is default
    assert ops._stream_of(5, device) is not default

    # a graph's host targets, prepared on the default stream and not yet fetched: the event
    # that they are kept for is one of that stream
    current, recorded = [], []

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    class Event:
        def record(self):
            recorded.append(current[-1])

        def query(self):
            return False

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    g = Graph.__new__(Graph)
    g.device, g._ctx = device, None
    g._prepares, g._copy_stream, g._copying, g._held = 0, None, collections.deque(), \
        collections.deque()
    for _ in range(65):
        g._hold_until_copied(object(), None)
    assert recorded == [default]
    g._hold_until_copied(object(), 7)  # another stream from here on
    assert recorded == [default, default]
    g._hold_until_copied(object(), None)
    assert recorded[2].cuda_stream == 7 and recorded[2].device == device


@pytest.mark.gpu
def test_a_call_is_ordered_by_the_default_stream_by_its_handle(cuda_device):
    table = torch.zeros(4_000_000, 64, device=cuda_device)
    ids = torch.full((100_000,), 3_999_999, dtype=torch.int32, device=cuda_device)
    torch.cuda.synchronize()
    for v in range(1, 9):
        table.fill_(v)
    got = ops.embedding_lookup(table, ids, stream=0)
    table.fill_(-1)
    assert float(got.sum()) == 8 * 64 * 100_000
    ops.check()


def test_a_graphs_default_stream_is_its_devices(monkeypatch):
    """Without a GPU: whatever device is current, as for prepare."""
    from paper_2601_01473_gb300 import agnes
    seen = []

    class Lib:
        def agnes_wait_hyperbatches(self, ctx, handle):
            seen.append(handle)
            return 0

        def agnes_sage_mean_layer(self, *args):
            seen.append(args[-1])
            return 0

    device = torch.device("cuda", 1)
    monkeypatch.setattr(agnes, "lib", Lib)
    monkeypatch.setattr(torch.cuda, "Stream", _Stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: _Stream(9 if d == device else 4))
    g = Graph.__new__(Graph)
    g.device, g._ctx = device, None
    g.fetch_all = lambda: type("Hyperbatch", (), {"node_size": torch.ones(2, 3)})
    g.wait()
    g.sage_mean_layer(0, torch.zeros(3, 2, 4), torch.zeros(2, 8, dtype=torch.float16))
    assert seen == [9, 9]
    g.wait(_Stream(6, device))
    assert seen[2] == 6
