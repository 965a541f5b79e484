"""The calls on rows of logits as programs make them: inside a network's gradient, one after the other, on other streams, captured
into graphs, with tensors that they have to refuse."""
import numpy as np
import pytest
import torch

import oracle as framework_oracle
import workloads
from gpu_util import normwise, to_dev, to_host
from oracle import logits as oracle

pytestmark = pytest.mark.gpu
F = np.float32


def forward(dims, w, X):
    """Layer inputs and logits of one worker in 64 bits; the smallest |z| / max|z| of any hidden unit."""
    a, acts, near = X.astype(np.float64), [X.astype(np.float64)], np.inf
    sl = framework_oracle.layer_slices(dims)
    for l, (ws, bs) in enumerate(sl):
        z = a @ w[ws].astype(np.float64).reshape(dims[l], dims[l + 1]) + w[bs].astype(np.float64)
        if l == len(sl) - 1:
            return acts, z, near
        near = min(near, np.abs(z).min() / np.abs(z).max())
        a = np.maximum(z, 0.0)
        acts.append(a)


def gradient(dims, w, X, dz):
    """Packed gradient of one worker from that of its logits."""
    acts, _, _ = forward(dims, w, X)
    sl = framework_oracle.layer_slices(dims)
    g = np.zeros(sl[-1][1].stop)
    for l in range(len(sl) - 1, -1, -1):
        ws, bs = sl[l]
        g[ws], g[bs] = (acts[l].T @ dz).ravel(), dz.sum(axis=0)
        if l:
            dz = (dz @ w[ws].astype(np.float64).reshape(dims[l], dims[l + 1]).T) * (acts[l] > 0)
    return g


def network(dims, P, b, seed):
    N = workloads.mlp_num_params(dims)
    wl = workloads.Workload("t", P=P, eta=0.05, rho=0.1, rounds=1, dims=tuple(dims), batch=b, N=N)
    ld = workloads.round_up(N, 4) + 4
    W = workloads.replicate(workloads.init_packed_weights(wl, seed=seed), P, ld)
    W[:, :N] += (np.random.default_rng(seed).standard_normal((P, N)) * 0.02).astype(F)
    X, y = workloads.minibatch(wl, 0, seed=seed)
    return N, ld, W, X, y


@pytest.mark.parametrize("dims, P, b, k, tail, hard, T, seed", [
    ((20, 10), 3, 7, 4, False, 0.0, 1.0, 1), ((20, 10), 1, 1, 10, True, 0.5, 2.0, 2), ((30, 17, 5), 4, 9, 3, True, 0.25, 4.0, 3),
    ((50, 24, 18, 100), 2, 12, 10, False, 0.5, 3.0, 4), ((300, 64, 1000), 2, 16, 20, True, 0.1, 2.0, 5), ((40, 16, 12), 5, 6, 16, False, 1.0, 1.0, 6)])
def test_gradient_of_a_network(dims, P, b, k, tail, hard, T, seed):
    import paper_1708_02983_amd as hip
    N, ld, W, X, y = network(dims, P, b, seed)
    C = dims[-1]
    rng = np.random.default_rng(seed + 100)
    idx = np.full((P, b, k), -1, np.int32)
    for p in range(P):
        for r in range(b):
            n = min(k, C)
            idx[p, r, :n] = rng.choice(C, n, replace=False)
    val = rng.normal(2.0, 2.0, (P, b, k)).astype(F)
    lse = (np.log(np.exp(np.where(idx >= 0, val, -np.inf) / T).sum(axis=2)) + 0.3).astype(F)
    labels = y.astype(np.int32)
    if b > 3:
        labels[0, 2] = -1
    G = torch.full((P, ld), float("nan"), device="cuda")
    loss = torch.empty(P, device="cuda")
    hip.easgd_grad_distill(dims, to_dev(W), to_dev(X), to_dev(idx), to_dev(val), G, loss=loss, temperature=T, teacher_lse=to_dev(lse) if tail else None,
                           labels=to_dev(labels) if hard else None, hard=hard)
    G, loss = to_host(G), to_host(loss)
    assert np.isnan(G[:, N:]).all()
    ref = np.full((P, ld), np.nan)
    for p in range(P):
        _, z, near = forward(dims, W[p], X[p])
        assert near > 1e-5, "a hidden unit within rounding of zero: choose another seed"
        dz, total = np.zeros_like(z), 0.0
        for r in range(b):
            l, g = oracle.distill(z[r], idx[p, r], val[p, r], np.float64(lse[p, r]) if tail else None, int(labels[p, r]) if hard else None, T, float(F(hard)))
            dz[r], total = g / b, total + l
        ref[p, :N] = gradient(dims, W[p], X[p], dz)
        # sums of at most 1001 fp32 terms a layer, three layers: the bound of the framework's other gradients
        assert abs(loss[p] - total / b) <= 1e-5 * max(1.0, abs(total / b))
    assert normwise(G, ref) <= 1e-5


def test_refusals_of_the_network_call():
    import paper_1708_02983_amd as hip
    dims, P, b, k = (20, 10), 2, 4, 3
    N, ld, W, X, y = network(dims, P, b, 1)
    dW, dX = to_dev(W), to_dev(X)
    idx, val = torch.zeros(P, b, k, dtype=torch.int32, device="cuda"), torch.zeros(P, b, k, device="cuda")
    G = torch.zeros_like(dW)
    with pytest.raises(ValueError, match="indices"):
        hip.easgd_grad_distill(dims, dW, dX, idx[:, :2], val, G)
    with pytest.raises(hip.EasgdError, match="hard = 0.5 needs labels"):
        hip.easgd_grad_distill(dims, dW, dX, idx, val, G, hard=0.5)
    with pytest.raises(hip.EasgdError, match="temperature"):
        hip.easgd_grad_distill(dims, dW, dX, idx, val, G, temperature=0.0)
    with pytest.raises(hip.EasgdError, match="at most 1024 classes"):
        wide = (20, 1025)
        n = workloads.round_up(workloads.mlp_num_params(wide), 4)
        hip.easgd_grad_distill(wide, torch.zeros(P, n, device="cuda"), dX, idx, val, torch.zeros(P, n, device="cuda"))


def test_a_round_of_learning_from_the_center():
    """The center scores the workers' minibatches, its top logits go to the workers, they take a step on them and exchange;
    a student's tokens are drawn from its logits.  Every stage against 64 bits from the stage before."""
    import paper_1708_02983_amd as hip
    dims, P, b, k, T = (60, 32, 40), 3, 10, 8, 2.0
    N, ld, W, X, y = network(dims, P, b, 11)
    Wc = (W[:, :N].mean(axis=0) + np.random.default_rng(3).standard_normal(N).astype(F) * F(0.01)).astype(F)
    dW, dWc, dX = to_dev(W), to_dev(Wc), to_dev(X)
    # the center's logits of all samples, layer by layer
    rows = P * b
    hidden = torch.empty(1, rows, dims[1], device="cuda")
    logits = torch.empty(1, rows, dims[2], device="cuda")
    n0 = (dims[0] + 1) * dims[1]
    c0, c1 = dWc[:n0].reshape(1, -1).contiguous(), dWc[n0:].reshape(1, -1).contiguous()
    hip.easgd_layer_product(0, dims[0], dims[1], dX.reshape(1, rows, dims[0]), hidden, Wl=c0, ld=c0.shape[1], out_ws=rows * dims[1], relu=True)
    hip.easgd_layer_product(0, dims[1], dims[2], hidden, logits, Wl=c1, ld=c1.shape[1], out_ws=rows * dims[2])
    logits = logits[0]
    z = np.stack([forward(dims, Wc, X.reshape(rows, -1))[1][r] for r in range(rows)])
    assert normwise(to_host(logits), z) <= 1e-5
    values, indices, lse = hip.easgd_top_logits(logits, k, temperature=T)
    z32 = to_host(logits).astype(np.float64)
    for r in range(rows):
        v, i, l = oracle.top_logits(z32[r], k, T)
        np.testing.assert_array_equal(to_host(indices)[r], i)
        assert abs(to_host(lse)[r] - l) <= 1e-5
    G = torch.zeros_like(dW)
    loss = torch.empty(P, device="cuda")
    shape = (P, b, k)
    hip.easgd_grad_distill(dims, dW, dX, indices.reshape(shape), values.reshape(shape), G, loss=loss, temperature=T, teacher_lse=lse.reshape(P, b))
    iv, vv, lv = to_host(indices).reshape(shape), to_host(values).reshape(shape), to_host(lse).reshape(P, b)
    ref = np.zeros((P, N))
    for p in range(P):
        _, zp, near = forward(dims, W[p], X[p])
        assert near > 1e-5
        dz = np.stack([oracle.distill(zp[r], iv[p, r], vv[p, r], np.float64(lv[p, r]), None, T, 0.0)[1] for r in range(b)]) / b
        ref[p] = gradient(dims, W[p], X[p], dz)
        # the same from the two-call form: a worker's logits, their loss and gradient
        zd = torch.from_numpy(zp.astype(F)).cuda()
        l2, g2 = hip.easgd_distill(zd, indices.reshape(shape)[p].contiguous(), values.reshape(shape)[p].contiguous(), temperature=T,
                                   teacher_lse=lse.reshape(P, b)[p].contiguous(), scale=1.0 / b)
        assert normwise(to_host(g2), dz) <= 2e-5 and abs(to_host(l2).mean() - to_host(loss)[p]) <= 2e-5
        u = np.random.default_rng(p).random(b).astype(F)
        tokens, logprob = hip.easgd_sample_tokens(zd, to_dev(u), temperature=torch.full((b,), T, device="cuda"))
        for r in range(b):
            token, lp, gap = oracle.sample_token(zp[r].astype(F), u[r], T)
            assert gap > 1e-8 and to_host(tokens)[r] == token and abs(to_host(logprob)[r] - lp) <= 1e-6
    assert normwise(to_host(G)[:, :N], ref) <= 1e-5
    hip.easgd_sync_round(dW, G, dWc, 0.05, 0.1, N=N)
    Wr, Wcr = W.copy(), Wc.copy()
    framework_oracle.easgd_round(Wr, to_host(G), Wcr, F(0.05), F(0.1), N=N)
    assert normwise(to_host(dW)[:, :N], Wr[:, :N]) <= 1e-5 and normwise(to_host(dWc), Wcr) <= 1e-5


def calls(rows, V, dtype, seed):
    """Inputs of one call of each kind, and a function that makes the calls and returns all that they put out."""
    import paper_1708_02983_amd as hip
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(rows, V, generator=gen, device="cuda") * 2).to(dtype)
    u = torch.rand(rows, generator=gen, device="cuda")
    p = torch.full((rows,), 0.9, device="cuda")
    k = torch.full((rows,), min(V, 400), dtype=torch.int32, device="cuda")
    labels = torch.randint(-1, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)

    def make(stream=None):
        values, indices, lse = hip.easgd_top_logits(z, min(V, 20), temperature=1.5, stream=stream)
        kw = dict(temperature=1.5, teacher_lse=lse + 0.1 if stream is None else lse, labels=labels, hard=0.25, stream=stream)
        loss, state = hip.easgd_distill_loss(z, indices, values, **kw)
        grad = hip.easgd_distill_grad(z, indices, values, state, scale=32.0, **kw)
        loss2, grad2 = hip.easgd_distill(z, indices, values, scale=32.0, **kw)
        out = [values, indices, lse, loss, state, grad, loss2, grad2]
        for filters in (dict(), dict(top_p=p), dict(top_k=k), dict(top_k=k, top_p=p, min_p=p * 0.05)):
            out += hip.easgd_sample_tokens(z, u, stream=stream, **filters)
        return out
    return z, u, make


def same(a, b):
    return all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) for x, y in zip(a, b))


@pytest.mark.parametrize("rows, V, dtype", [(5, 100, torch.float32), (300, 3000, torch.bfloat16), (3, 100001, torch.float16)])
def test_graphs(rows, V, dtype):
    """Captured once, replayed on new inputs with eager work between the replays: the eager results every time."""
    z, u, make = calls(rows, V, dtype, 1)
    make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = make()
    for turn in range(4):
        z.copy_((torch.randn(rows, V, device="cuda") * (1 + turn)).to(dtype))
        u.uniform_()
        eager = [t.clone() for t in make()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(captured, eager), turn


def test_two_graphs_and_two_streams_at_once():
    """Graphs with workspaces of their own replayed side by side, and eager calls on two streams, disturb nobody."""
    sets = [calls(4, 70000, torch.bfloat16, seed) for seed in (1, 2)]
    expected = [[t.clone() for t in make()] for _, _, make in sets]
    torch.cuda.synchronize()
    graphs, captured = [], []
    for _, _, make in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured.append(make())
        graphs.append(graph)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert same(captured[0], expected[0]) and same(captured[1], expected[1])
        got = []
        for (_, _, make), stream in zip(sets, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                got.append(make())
        torch.cuda.synchronize()
        assert same(got[0], expected[0]) and same(got[1], expected[1])


def test_a_stream_given_by_hand():
    z, u, make = calls(3, 90000, torch.float32, 5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = make(stream=side)
    side.synchronize()
    with torch.cuda.stream(side):
        again = make(stream=side)
    side.synchronize()
    assert same(got, again)


def test_results_are_written_where_asked_and_nowhere_else():
    import paper_1708_02983_amd as hip
    rows, V, k = 7, 5000, 9
    z = torch.randn(rows, V, device="cuda").to(torch.float16)
    buf = torch.full((rows + 2, k), 5.5, device="cuda")
    ibuf = torch.full((rows + 2, k), 77, dtype=torch.int32, device="cuda")
    l = torch.full((rows + 2,), 5.5, device="cuda")
    values, indices, lse = hip.easgd_top_logits(z, k, values=buf[1:-1], indices=ibuf[1:-1], lse=l[1:-1])
    ref = hip.easgd_top_logits(z, k)
    assert torch.equal(values, ref[0]) and torch.equal(indices, ref[1]) and torch.equal(lse, ref[2])
    for t, v in ((buf, 5.5), (ibuf, 77), (l, 5.5)):
        assert (t[0] == v).all() and (t[-1] == v).all()
    tok = torch.full((rows + 2,), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((rows + 2,), 5.5, device="cuda")
    u = torch.rand(rows, device="cuda")
    hip.easgd_sample_tokens(z, u, tokens=tok[1:-1], logprob=lp[1:-1])
    assert torch.equal(tok[1:-1], hip.easgd_sample_tokens(z, u)[0]) and tok[0] == 77 and tok[-1] == 77 and lp[0] == 5.5 and lp[-1] == 5.5


def test_refused_tensors():
    import paper_1708_02983_amd as hip
    z = torch.randn(6, 50, device="cuda")
    idx, val = torch.zeros(6, 4, dtype=torch.int32, device="cuda"), torch.zeros(6, 4, device="cuda")
    u = torch.rand(6, device="cuda")
    with pytest.raises(ValueError, match="follow one another"):
        hip.easgd_top_logits(z.t(), 3)
    with pytest.raises(ValueError, match="overlap"):
        hip.easgd_top_logits(z[:1].expand(6, 50), 3)
    with pytest.raises(ValueError, match=r"\[rows\]\[V\]"):
        hip.easgd_top_logits(z[0], 3)
    with pytest.raises(TypeError, match="float32"):
        hip.easgd_top_logits(z.double(), 3)
    with pytest.raises(ValueError, match="k must be"):
        hip.easgd_top_logits(z, 257)
    with pytest.raises(TypeError, match="indices must be torch.int32"):
        hip.easgd_distill(z, idx.long(), val)
    with pytest.raises(ValueError, match="values must be contiguous"):
        hip.easgd_distill(z, idx, val[:5])
    with pytest.raises(ValueError, match="dlogits must be"):
        hip.easgd_distill(z, idx, val, dlogits=torch.empty(6, 51, device="cuda"))
    with pytest.raises(ValueError, match="labels must be"):
        hip.easgd_distill(z, idx, val, labels=torch.zeros(5, dtype=torch.int32, device="cuda"), hard=0.5)
    with pytest.raises(TypeError, match="u must be a CUDA/HIP tensor"):
        hip.easgd_sample_tokens(z, u.cpu())
    with pytest.raises(TypeError, match="top_k must be torch.int32"):
        hip.easgd_sample_tokens(z, u, top_k=u)
    with pytest.raises(ValueError, match="workspace holds"):
        big = torch.randn(2, 200000, device="cuda")
        hip.easgd_top_logits(big, 4, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(hip.EasgdError, match="temperature"):
        hip.easgd_top_logits(z, 3, temperature=0.0)
    with pytest.raises(hip.EasgdError, match="V \\(1048577\\) above"):
        hip.easgd_top_logits(torch.zeros(1, (1 << 20) + 1, device="cuda"), 3)


def test_rows_far_into_memory():
    """Rows whose offsets pass 2^31 and 2^32 elements: a stride of 2^26 elements over 70 rows.  The near copy's rows start on the
    same 16-byte grid, so that sums have the same order."""
    import paper_1708_02983_amd as hip
    rows, V, ld = 70, 1500, 1 << 26
    buf = torch.empty((rows - 1) * ld + V + 4096, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((rows, V), (ld, 1))
    small = torch.randn(rows, 1504, device="cuda").to(torch.bfloat16)[:, :V]
    z.copy_(small)
    a, b = hip.easgd_top_logits(z, 30), hip.easgd_top_logits(small, 30)
    assert same(a, b)
    u = torch.rand(rows, device="cuda")
    assert same(hip.easgd_sample_tokens(z, u), hip.easgd_sample_tokens(small, u))
    # the gradient back into the same far rows' neighbours
    out = buf.as_strided((rows, V), (ld, 1), 4096)
    l1, g1 = hip.easgd_distill(z, b[1], b[0], dlogits=out, scale=8.0)
    l2, g2 = hip.easgd_distill(small, b[1], b[0], scale=8.0)
    assert torch.equal(l1, l2) and torch.equal(g1, g2)
