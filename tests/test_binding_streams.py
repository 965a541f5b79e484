"""Whose memory the binding's results and workspaces are when a call gets a stream (no GPU needed: the allocator is a stand-in)."""
import contextlib
import os

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_1708_02983_amd", "libeasgd_hip.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libeasgd_hip.so not built (run __graft_entry__.build())")


class Machine:
    """Streams, the current one, and an allocator that notes in whose pool a tensor was made and who else uses it."""

    def __init__(self, monkeypatch):
        import paper_1708_02983_amd.binding as binding
        self.current, self.made = "caller", []
        machine = self

        class Tensor:
            def __init__(self):
                self.pool, self.users = machine.current, []

            def record_stream(self, stream):
                self.users.append(stream)

        def empty(*args, **kw):
            self.made.append(Tensor())
            return self.made[-1]

        @contextlib.contextmanager
        def use(stream):
            before, self.current = self.current, stream
            yield
            self.current = before

        self.binding = binding
        monkeypatch.setattr(torch, "empty", empty)
        monkeypatch.setattr(torch.cuda, "stream", use)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(binding, "_stream_object", lambda s: s, raising=False)


class Like:
    device = "cuda:0"


def test_results_belong_to_the_stream_that_writes_them(monkeypatch):
    """Memory that the caller's stream has just given back may still be read or written by that stream's work, which the other stream does not
    wait for: it must not come back as the other stream's result."""
    m = Machine(monkeypatch)
    t = m.binding._new((3,), torch.float32, Like, "side")
    assert t.pool == "side" and t.users == ["caller"] and m.current == "caller"


def test_the_callers_own_stream(monkeypatch):
    m = Machine(monkeypatch)
    for stream in (None, "caller"):
        t = m.binding._new((3,), torch.float32, Like, stream)
        assert t.pool == "caller" and t.users == []


@pytest.mark.parametrize("call", ["easgd_grad", "easgd_mlp_round"])
def test_workspaces_of_the_network_calls(monkeypatch, call):
    m = Machine(monkeypatch)
    dims = (20, 10)
    W, X, y = torch.zeros(2, 212), torch.zeros(2, 3, 20), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(TypeError, match="CUDA/HIP"):          # the tensors are on no GPU: refused, with the workspace made
        if call == "easgd_grad":
            m.binding.easgd_grad(dims, W, X, y, W, stream="side")
        else:
            m.binding.easgd_mlp_round(dims, W, W, X, y, 0.1, 0.1, stream="side")
    assert [t.pool for t in m.made] == ["side"] and m.made[0].users == ["caller"]


def test_a_stream_of_another_device(monkeypatch):
    """Kernels on it would run on a device that does not have the tensors."""
    from paper_1708_02983_amd import binding

    class Stream:
        cuda_stream = 5

        def __init__(self, device):
            self.device = device

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="stream is on cuda:1, the current device is cuda:0"):
        binding._stream(Stream(torch.device("cuda:1")))
    assert binding._stream(Stream(torch.device("cuda:0"))).value == 5
    assert binding._stream(Stream("anything")).value == 5
