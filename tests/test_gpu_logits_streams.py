"""Calls on rows of logits that get a stream: their results' memory, and their place in a graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def inputs(rows, V, k):
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(rows, V, generator=gen, device="cuda")
    idx = torch.randint(0, V, (rows, k), generator=gen, device="cuda", dtype=torch.int32)
    return z, idx, torch.randn(rows, k, generator=gen, device="cuda"), torch.rand(rows, generator=gen, device="cuda")


def test_results_are_not_memory_that_the_current_stream_still_writes():
    import paper_1708_02983_amd as hip
    rows, V, k = 300, 50000, 5
    z, idx, val, u = inputs(rows, V, k)
    expected = [t.clone() for t in (*hip.easgd_distill(z, idx, val), *hip.easgd_sample_tokens(z, u))]
    side = torch.cuda.Stream()
    a = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(20):
        a = a @ a * 1e-4                               # work for a while, at whose end the block is written
    block = torch.empty(rows, V, device="cuda")
    block.fill_(7.0)
    where = block.data_ptr()
    del block                                          # free for the current stream only
    got = [*hip.easgd_distill(z, idx, val, stream=side), *hip.easgd_sample_tokens(z, u, stream=side)]
    assert got[1].data_ptr() != where
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, expected))


def test_a_branch_of_a_graph():
    """A call on a stream that forks from the captured one and joins it again, replayed on new inputs."""
    import paper_1708_02983_amd as hip
    z, idx, val, u = inputs(3, 70000, 8)
    side = torch.cuda.Stream()

    def make():
        side.wait_stream(torch.cuda.current_stream())
        there = [*hip.easgd_distill(z, idx, val, stream=side), *hip.easgd_top_logits(z, 8, stream=side)]
        here = [*hip.easgd_sample_tokens(z, u)]
        torch.cuda.current_stream().wait_stream(side)
        return there + here

    make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = make()
    for _ in range(3):
        z.normal_()
        u.uniform_()
        eager = [t.clone() for t in make()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(captured, eager))


def test_streams_that_are_only_a_handle():
    import paper_1708_02983_amd as hip

    class Handle:
        def __init__(self, stream):
            self.cuda_stream = stream.cuda_stream

    z, _, _, u = inputs(4, 500, 3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    tokens, _ = hip.easgd_sample_tokens(z, u, stream=Handle(side))
    side.synchronize()
    assert torch.equal(tokens, hip.easgd_sample_tokens(z, u)[0])


def test_replicas_of_another_device_than_the_current_one(monkeypatch):
    """Refused by name, before a workspace is made or anything is launched."""
    import paper_1708_02983_amd as hip
    dims, P, b, k = (20, 10), 2, 4, 3
    W, X = torch.zeros(P, 212, device="cuda"), torch.zeros(P, b, 20, device="cuda")
    idx, val = torch.zeros(P, b, k, dtype=torch.int32, device="cuda"), torch.zeros(P, b, k, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="W must be on cuda:1, is on cuda:0"):
        hip.easgd_grad_distill(dims, W, X, idx, val, W.clone())
    with pytest.raises(ValueError, match="logits is on cuda:0, the current device is cuda:1"):
        hip.easgd_distill(X[0], idx[0], val[0])
