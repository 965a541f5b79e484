"""The calls on given tokens and the AdamW rounds as programs make them: inside a network's gradient, one after the other, on other streams, captured into
graphs, far into memory, with tensors that they have to refuse."""
import numpy as np
import pytest
import torch

import workloads
from gpu_util import normwise, to_dev, to_host
from logits_util import sum_error
from oracle import adamw as oa
from oracle import tokens as ot
from test_gpu_logits_calls import forward, gradient, network

pytestmark = pytest.mark.gpu
F = np.float32


@pytest.fixture(scope="module")
def hip():
    import paper_1708_02983_amd as pkg
    return pkg


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b) if x is not None)


@pytest.mark.parametrize("dims, P, b, bonus, T, weighted, seed", [
    ((20, 10), 3, 7, 0.0, 1.0, False, 1), ((20, 10), 1, 1, 0.5, 2.0, True, 2), ((30, 17, 5), 4, 9, 0.1, 1.0, True, 3),
    ((50, 24, 18, 100), 2, 12, 0.0, 0.5, True, 4), ((300, 64, 1000), 2, 16, 0.25, 1.0, False, 5)])
def test_gradient_of_a_network(hip, dims, P, b, bonus, T, weighted, seed):
    N, ld, W, X, y = network(dims, P, b, seed)
    rng = np.random.default_rng(seed)
    tokens = y.astype(np.int32)
    if b > 3:
        tokens[0, 2] = -1
    weight = rng.normal(size=(P, b)).astype(F) if weighted else None
    G = torch.full((P, ld), float("nan"), device="cuda")
    loss, logprob, entropy = torch.empty(P, device="cuda"), torch.empty(P, b, device="cuda"), torch.empty(P, b, device="cuda")
    hip.easgd_grad_token_loss(dims, to_dev(W), to_dev(X), to_dev(tokens), G, loss=loss, weight=None if weight is None else to_dev(weight), bonus=bonus, temperature=T,
                              logprob=logprob, entropy=entropy)
    G = to_host(G)
    assert np.isnan(G[:, N:]).all()
    ref = np.full((P, ld), np.nan)
    for p in range(P):
        _, z, near = forward(dims, W[p], X[p])
        assert near > 1e-5, "a hidden unit within rounding of zero: choose another seed"
        dz, total = np.zeros_like(z), 0.0
        for r in range(b):
            token = int(tokens[p, r])
            l, g = ot.token_loss(z[r], token, 1.0 if weight is None else float(weight[p, r]), float(F(bonus)), T)
            dz[r], total = g / b, total + l
            lp, h, *_ = ot.score(z[r], token, T)
            # logits are sums of at most 301 terms: the bound of the framework's other gradients
            assert abs(logprob[p, r].item() - lp) <= 1e-5 * max(1.0, abs(lp)) and abs(entropy[p, r].item() - h) <= 1e-5 * max(1.0, h)
        ref[p, :N] = gradient(dims, W[p], X[p], dz)
        assert abs(loss[p].item() - total / b) <= 1e-5 * max(1.0, abs(total / b))
    assert normwise(G, ref) <= 1e-5


@pytest.mark.parametrize("eight", [False, True])
def test_answers_are_drawn_scored_and_learned_from(hip, eight):
    """The center answers, the answers are scored, every worker learns from them with weights and clipped gradients, and all exchange: three rounds,
    every stage against 64 bits (stored bits) from what the stage before left."""
    dims, P, b = (60, 32, 40), 3, 10
    N, ld, W, X, y = network(dims, P, b, 11)
    rows = P * b
    blocks = (N + 255) // 256
    rng = np.random.default_rng(4)
    dW, dWc, dX = to_dev(W), to_dev(W[:, :N].mean(axis=0)), to_dev(X)
    if eight:
        dM, dS = torch.zeros((P, ld), dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros((P, ld), dtype=torch.float8_e5m2, device="cuda")
        dMs, dSs = torch.zeros((P, blocks), device="cuda"), torch.zeros((P, blocks), device="cuda")
        more = dict(M_scale=dMs, S_scale=dSs, seed=3)
    else:
        dM, dS, more = torch.zeros((P, ld), device="cuda"), torch.zeros((P, ld), device="cuda"), {}
    l0 = (dims[0] + 1) * dims[1]
    l1 = N
    ends = torch.tensor([dims[0] * dims[1], l0, l0 + dims[1] * dims[2], l1], device="cuda")
    rates, decays = torch.tensor([1.0, 1.0, 0.5, 0.5], device="cuda"), torch.tensor([0.01, 0.0, 0.01, 0.0], device="cuda")
    G = torch.zeros_like(dW)
    for step in (1, 2, 3):
        hidden, logits = torch.empty(1, rows, dims[1], device="cuda"), torch.empty(1, rows, dims[2], device="cuda")
        c0, c1 = dWc[:l0].reshape(1, -1).contiguous(), dWc[l0:].reshape(1, -1).contiguous()
        hip.easgd_layer_product(0, dims[0], dims[1], dX.reshape(1, rows, dims[0]), hidden, Wl=c0, ld=c0.shape[1], out_ws=rows * dims[1], relu=True)
        hip.easgd_layer_product(0, dims[1], dims[2], hidden, logits, Wl=c1, ld=c1.shape[1], out_ws=rows * dims[2])
        tokens, drawn = hip.easgd_sample_tokens(logits[0], torch.from_numpy(rng.random(rows).astype(F)).cuda())
        scores = hip.easgd_score_tokens(logits[0], tokens, k=5, rank=True)
        z = to_host(logits)[0]
        for r in range(rows):
            lp, h, rank, top, places = ot.score(z[r], int(tokens[r]), 1.0, 5)
            assert abs(scores.logprob[r].item() - lp) <= 2e-6 and abs(scores.entropy[r].item() - h) <= 4e-6 and scores.rank[r].item() == rank
            assert scores.top_indices[r].tolist() == places.tolist()
        assert torch.allclose(scores.logprob, drawn, rtol=0, atol=4e-6)          # nothing was filtered
        weight = torch.from_numpy(rng.normal(size=(P, b)).astype(F)).cuda()
        before, before_c = to_host(dW), to_host(dWc)
        m, s = to_host(dM.float())[:, :N], to_host(dS.float())[:, :N]
        if eight:
            m, s = (x * np.repeat(to_host(sc), 256, axis=1)[:, :N] for x, sc in ((m, dMs), (s, dSs)))
        hip.easgd_grad_token_loss(dims, dW, dX, tokens.reshape(P, b), G, weight=weight, bonus=0.01)
        norm, clip = hip.easgd_grad_norms(G, max_norm=0.05, N=N)
        g = to_host(G)[:, :N]
        want, want_clip = oa.norms(g, 0.05)
        np.testing.assert_allclose(to_host(norm), want, rtol=2.0 ** -23)
        np.testing.assert_allclose(to_host(clip), want_clip, rtol=2.0 ** -23)
        hip.adamw_round(dW, dM, dS, G, step, 0.01, Wc=dWc, rho=0.1, tensors=(ends, rates, decays), clip=clip, N=N, **more)
        table = tuple(to_host(t) for t in (ends, rates, decays))
        w, c, m1, s1, size = oa.adamw_round(before[:, :N], m, s, g, before_c, step, 0.01, 0.1, tensors=table, clip=to_host(clip))
        assert (np.abs(to_host(dW)[:, :N] - w) <= 2.0 ** -24 * (np.abs(w) + 16 * size)).all()
        assert (np.abs(to_host(dWc) - c) <= 2.0 ** -24 * (np.abs(c) + 0.01 * (P + 4) * (np.abs(before[:, :N]).sum(axis=0) + P * np.abs(before_c)))).all()
        if eight:
            for i in range(P):
                codes = oa.encode(m1[i], s1[i], i, step, 3)
                for d, x in zip((dM.view(torch.uint8), dS.view(torch.uint8), dMs, dSs), codes):
                    assert np.array_equal(d[i, :len(x)].cpu().numpy(), x)
        else:
            assert np.array_equal(to_host(dM)[:, :N], m1) and np.array_equal(to_host(dS)[:, :N], s1)


def calls(hip, rows, V, dtype, seed):
    """Inputs and the calls on them, results as a flat list."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, V, generator=gen, device="cuda").to(dtype)
    tokens = torch.randint(-1, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    weight = torch.randn(rows, generator=gen, device="cuda")
    P, N = 5, 20001
    ld = 20004
    start = [torch.randn(P, ld, generator=gen, device="cuda") * 0.1 for _ in range(2)]
    g = torch.randn(P, ld, generator=gen, device="cuda") * 1e-3
    step, eta = torch.tensor([3], device="cuda"), torch.tensor([0.01], device="cuda")

    def make(stream=None):
        kw = {} if stream is None else {"stream": stream}
        with torch.cuda.stream(stream) if stream is not None else torch.cuda.stream(torch.cuda.current_stream()):
            W, Wc = start[0].clone(), start[1][0, :N].clone()
            W8, M, S = start[0].clone(), torch.zeros_like(W), torch.zeros_like(W)
            M8, S8 = torch.zeros((P, ld), device="cuda").to(torch.float8_e4m3fn), torch.zeros((P, ld), device="cuda").to(torch.float8_e5m2)
            Ms, Ss = torch.zeros((P, (N + 255) // 256), device="cuda"), torch.zeros((P, (N + 255) // 256), device="cuda")
        s = hip.easgd_score_tokens(z, tokens, k=6, rank=True, state=True, **kw)
        plain = hip.easgd_score_tokens(z, tokens, state=True, **kw)
        d = hip.easgd_score_tokens_grad(z, tokens, plain.state, dlogprob=weight, dentropy=weight, **kw)
        loss = hip.easgd_token_loss(z, tokens, weight=weight, bonus=0.1, scale=4.0, entropy=True, **kw)
        norm, clip = hip.easgd_grad_norms(g, max_norm=0.1, N=N, **kw)
        hip.adamw_round(W, M, S, g, step, eta, Wc=Wc, rho=0.1, clip=clip, N=N, **kw)
        hip.adamw_round(W8, M8, S8, g, step, eta, clip=clip, M_scale=Ms, S_scale=Ss, seed=9, N=N, **kw)
        return [*s, *plain[:2], d, *loss, norm, clip, W, Wc, M, S, W8, M8, S8, Ms, Ss]
    return z, tokens, weight, g, step, eta, make


@pytest.mark.parametrize("rows,V,dtype", [(5, 70, torch.float32), (40, 70001, torch.bfloat16), (300, 9000, torch.float16)])
def test_replays_with_eager_work_between(hip, rows, V, dtype):
    """A captured set of calls, replayed on inputs that changed (the step and the rate among them), with eager calls between the replays."""
    z, tokens, weight, g, step, eta, make = calls(hip, rows, V, dtype, 1)
    make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = make()
    for t in range(3):
        z.copy_(torch.randn(rows, V, device="cuda"))
        tokens.copy_(torch.randint(-1, V, (rows,), device="cuda"))
        weight.normal_()
        g.normal_(0.0, 1e-3)
        step.fill_(5 + t)
        eta.fill_(0.01 / (t + 1))
        eager = [None if x is None else x.clone() for x in make()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(eager, captured), t


def test_two_graphs_side_by_side_and_two_streams(hip):
    sets = [calls(hip, 40, 70001, torch.bfloat16, 1), calls(hip, 280, 20000, torch.float32, 2)]
    expected, graphs, captured = [], [], []
    for *_, make in sets:
        expected.append([None if x is None else x.clone() for x in make()])
        torch.cuda.synchronize()
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
        for (*_, make), stream in zip(sets, streams):
            stream.wait_stream(torch.cuda.current_stream())
            got.append(make(stream))
        torch.cuda.synchronize()
        assert same(got[0], expected[0]) and same(got[1], expected[1])


def test_rows_far_into_memory(hip):
    """Rows whose offsets pass 2^31 and 2^32 elements, on the same 16-byte grid as the near copy's, so that sums have the same order."""
    rows, V, ld = 70, 1500, 1 << 26
    buf = torch.empty((rows - 1) * ld + V + 4096, dtype=torch.bfloat16, device="cuda")
    z = buf.as_strided((rows, V), (ld, 1))
    small = torch.randn(rows, 1504, device="cuda").to(torch.bfloat16)[:, :V]
    z.copy_(small)
    tokens = torch.randint(-1, V, (rows,), device="cuda", dtype=torch.int32)
    assert same(hip.easgd_score_tokens(z, tokens, k=30, rank=True, state=True), hip.easgd_score_tokens(small, tokens, k=30, rank=True, state=True))
    assert same(hip.easgd_score_tokens(z, tokens, rank=True), hip.easgd_score_tokens(small, tokens, rank=True))
    out = buf.as_strided((rows, V), (ld, 1), 4096)
    one, two = hip.easgd_token_loss(z, tokens, bonus=0.5, dlogits=out, scale=8.0), hip.easgd_token_loss(small, tokens, bonus=0.5, scale=8.0)
    assert same(one, two)
    state = hip.easgd_score_tokens(small, tokens, state=True).state
    ones = torch.ones(rows, device="cuda")
    assert same([hip.easgd_score_tokens_grad(z, tokens, state, dentropy=ones, dlogits=out)], [hip.easgd_score_tokens_grad(small, tokens, state, dentropy=ones)])
    # replicas: the last of 66 rows of 2^26 gradients starts behind 2^32 elements
    g = torch.zeros((66, 1 << 26), dtype=torch.bfloat16, device="cuda")
    g[65, :300] = torch.randn(300, device="cuda")
    norm, clip = hip.easgd_grad_norms(g, max_norm=1.0)
    assert not norm[:65].any() and torch.isclose(norm[65], g[65, :300].double().norm().float())
    assert hip.easgd_grad_norms(g, max_norm=1.0, N=300)[0][65] == norm[65]


def test_replicas_far_into_memory(hip):
    """AdamW on a few parameters of rows that lie 2^27 elements apart, against the same rows packed."""
    P, N, ld = 34, 1000, 1 << 27
    gen = torch.Generator(device="cuda").manual_seed(4)
    near = [torch.randn(P, N, generator=gen, device="cuda") * 0.01 for _ in range(2)]
    far = []
    for x in near:
        t = torch.zeros((P, ld), dtype=torch.float32, device="cuda")
        t[:, :N] = x
        far.append(t)
    results = []
    for W, G, l in ((near[0].clone(), near[1], N), (far[0], far[1], ld)):
        M8, S8 = torch.zeros((P, l), dtype=torch.uint8, device="cuda"), torch.zeros((P, l), dtype=torch.uint8, device="cuda")
        Ms, Ss = torch.zeros((P, 4), device="cuda"), torch.zeros((P, 4), device="cuda")
        Wc = near[0].mean(dim=0)
        for step in (1, 2):
            hip.adamw_round(W, M8.view(torch.float8_e4m3fn), S8.view(torch.float8_e5m2), G, step, 0.01, Wc=Wc, rho=0.1, M_scale=Ms, S_scale=Ss, N=N)
        results.append([W[:, :N].clone(), M8[:, :N].clone(), S8[:, :N].clone(), Ms, Ss, Wc])
        del M8, S8
    assert same(*results)


def test_results_are_written_where_asked_and_nowhere_else(hip):
    rows, V, k = 7, 5000, 9
    z = torch.randn(rows, V, device="cuda").to(torch.float16)
    tokens = torch.randint(0, V, (rows,), device="cuda", dtype=torch.int32)
    ref = hip.easgd_score_tokens(z, tokens, k=k, rank=True, state=True)
    bufs = [torch.full((rows + 2, *t.shape[1:]), 77, dtype=t.dtype, device="cuda") for t in ref]
    got = hip.easgd_score_tokens(z, tokens, k=k, **{n: b[1:-1] for n, b in zip(ref._fields, bufs)})
    assert same(got, ref) and all((b[0] == 77).all() and (b[-1] == 77).all() for b in bufs)
    none = hip.easgd_score_tokens(z, tokens, entropy=None)
    assert none.entropy is None and none.rank is None and none.state is None and none.top_indices is None
    # with alternatives a row is summed in another order: each sum is within sum_error of the exact one, and each logprob (below 16) rounded once
    assert (none.logprob.double() - ref.logprob.double()).abs().max().item() <= 2 * sum_error(V) + 2 * 2.0 ** -24 * 16
    empty = hip.easgd_score_tokens(z[:0], tokens[:0], k=2, rank=True)
    assert empty.logprob.shape == (0,) and empty.top_indices.shape == (0, 2)
    assert hip.easgd_token_loss(z[:0], tokens[:0])[3].shape == (0, V)


def test_refused_tensors(hip):
    z = torch.randn(6, 50, device="cuda")
    t = torch.zeros(6, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="follow one another"):
        hip.easgd_score_tokens(z.t(), t)
    with pytest.raises(TypeError, match="tokens must be torch.int32"):
        hip.easgd_score_tokens(z, t.long())
    with pytest.raises(ValueError, match="tokens must be contiguous"):
        hip.easgd_token_loss(z, t[:5])
    with pytest.raises(ValueError, match="k must be"):
        hip.easgd_score_tokens(z, t, k=257)
    with pytest.raises(ValueError, match="need k > 0"):
        hip.easgd_score_tokens(z, t, top_logprob=z)
    with pytest.raises(hip.EasgdError, match="need tokens"):
        hip.easgd_score_tokens(z, rank=True)
    with pytest.raises(hip.EasgdError, match="must not overlap"):
        hip.easgd_token_loss(z, t, dlogits=z)
    with pytest.raises(hip.EasgdError, match="NULL pointer"):
        hip.easgd_score_tokens_grad(z, t, torch.zeros(6, 4, device="cuda"))
    with pytest.raises(hip.EasgdError, match="bonus"):
        hip.easgd_token_loss(z, t, bonus=float("nan"))
    W, M, S = (torch.zeros(2, 8, device="cuda") for _ in range(3))
    with pytest.raises(TypeError, match="W must be torch.float32"):
        hip.adamw_round(W.bfloat16(), M, S, W, 1, 0.1)
    with pytest.raises(ValueError, match="G must be"):
        hip.adamw_round(W, M, S, torch.zeros(3, 8, device="cuda"), 1, 0.1)
    with pytest.raises(TypeError, match="S must be torch.float8_e5m2"):
        hip.adamw_round(W, M.to(torch.float8_e4m3fn), S.to(torch.float8_e4m3fn), W, 1, 0.1)
    with pytest.raises(ValueError, match="need M_scale"):
        hip.adamw_round(W, M.to(torch.float8_e4m3fn), S.to(torch.float8_e5m2), W, 1, 0.1)
    with pytest.raises(ValueError, match="belong to moments in 8 bits"):
        hip.adamw_round(W, M, S, W, 1, 0.1, M_scale=W)
    with pytest.raises(ValueError, match=r"N must be in \[1, 8\]"):
        hip.adamw_round(W, M, S, W, 1, 0.1, N=9)
    with pytest.raises(hip.EasgdError, match="needs a center"):
        hip.adamw_round(W, M, S, W, 1, 0.1, rho=0.5)
    with pytest.raises(hip.EasgdError, match="step must be >= 1"):
        hip.adamw_round(W, M, S, W, 0, 0.1)
    with pytest.raises(TypeError, match="ends must be torch.int64"):
        hip.adamw_round(W, M, S, W, 1, 0.1, tensors=(t, z[0, :6], z[0, :6]))
    with pytest.raises(ValueError, match="must be contiguous"):
        hip.easgd_grad_norms(torch.zeros(8, 2, device="cuda").t())
    with pytest.raises(hip.EasgdError, match="max_norm"):
        hip.easgd_grad_norms(W, max_norm=0.0)
