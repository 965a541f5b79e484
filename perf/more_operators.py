"""The operators of learning from given tokens that are timed, and the ranges that they stand for.

  * ``easgd_score_tokens``: the log probability of a given token of every row of logits, the row's entropy, the token's rank and
    the row's first alternatives (kind "score");
  * ``easgd_score_tokens_grad``: the gradient of log probabilities and entropies, from what the forward pass left (kind "score_grad");
  * ``easgd_token_loss``: weighted negative log probabilities less an entropy bonus, and their gradient, in one call (kind "token_loss");
  * ``easgd_grad_norms``: the norm of every worker's gradient and the factor that clips it (kind "norms");
  * ``adamw_round``: an AdamW step of all replicas over all tensors, with or without the elastic exchange, its moments in 32 bits
    (kind "adamw") or in 8 (kind "adamw8").

With ``own`` false ``run`` computes the same from elementary torch operations.  ``rows`` counts rows of logits, ``V`` is their length;
``P`` counts workers, ``N`` a replica's parameters.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
NEG = float("-inf")
BLOCK = 256                                     # parameters that share a scale in 8 bits


def listed():
    return [
        # the log probabilities of a training batch's tokens under a large vocabulary, with entropies and ranks: the largest read
        {"name": "score_batch", "kind": "score", "rows": 2048, "V": 131072, "ld": "packed", "dtype": "bf16", "k": 0, "T": 1.0,
         "rank": True, "padding": 128},
        # a server that answers with the log probabilities of its tokens and twenty alternatives each, an odd vocabulary
        {"name": "score_alternatives", "kind": "score", "rows": 48, "V": 50001, "ld": "packed", "dtype": "fp16", "k": 20, "T": 0.8,
         "rank": True, "padding": 0},
        # backward alone, for a program that makes its loss of the log probabilities and entropies itself
        {"name": "score_backward", "kind": "score_grad", "rows": 1024, "V": 32000, "ld": "padded", "dtype": "bf16", "T": 1.0,
         "entropy": True, "padding": 64},
        # the framework's own networks: sixteen workers, 128 samples, a hundred classes: launches and latency
        {"name": "score_backward_classes", "kind": "score_grad", "rows": 2048, "V": 100, "ld": "packed", "dtype": "fp32", "T": 2.0,
         "entropy": False, "padding": 0},
        # learning from answers with weights and an entropy bonus, loss and gradient in one call: padded positions
        {"name": "token_loss_batch", "kind": "token_loss", "rows": 2048, "V": 131072, "ld": "packed", "dtype": "bf16", "T": 1.0,
         "bonus": 0.01, "padding": 128},
        # plain likelihood of an odd vocabulary
        {"name": "token_loss_odd", "kind": "token_loss", "rows": 777, "V": 50001, "ld": "packed", "dtype": "fp16", "T": 1.0,
         "bonus": 0.0, "padding": 0},
        # eight replicas of 61 M parameters: the norms that clip their gradients
        {"name": "norms_large", "kind": "norms", "P": 8, "N": 61000000, "ld": "padded", "dtype": "fp32", "max_norm": 1.0},
        # sixteen workers of 784-1024-1024-10, gradients stored in 16 bits
        {"name": "norms_mlp", "kind": "norms", "P": 16, "N": 1863690, "ld": "padded", "dtype": "bf16", "max_norm": 1.0},
        # a local step of eight replicas of 61 M parameters: the largest of all
        {"name": "adamw_large", "kind": "adamw", "P": 8, "N": 61000000, "ld": "padded", "dtype": "fp32", "elastic": False, "tensors": 16,
         "clip": True, "step": 1000},
        # sixteen workers of 784-1024-1024-10 with the elastic exchange, weights decayed and biases not, gradients in 16 bits
        {"name": "adamw_mlp", "kind": "adamw", "P": 16, "N": 1863690, "ld": "padded", "dtype": "bf16", "elastic": True, "tensors": 6,
         "clip": True, "step": 17},
        # the same replicas as the largest with their moments in 8 bits and the elastic exchange
        {"name": "adamw8_large", "kind": "adamw8", "P": 8, "N": 61000000, "ld": "padded", "dtype": "fp32", "elastic": True, "tensors": 16,
         "clip": False, "step": 1000},
        # four workers of softmax regression 784-10: launches and latency
        {"name": "adamw8_small", "kind": "adamw8", "P": 4, "N": 7850, "ld": "padded", "dtype": "fp32", "elastic": True, "tensors": 2,
         "clip": True, "step": 3},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("score", "score", "score_grad", "token_loss", "token_loss", "norms", "adamw", "adamw", "adamw8", "adamw8"))
    if kind in ("score", "score_grad", "token_loss"):
        case = {"kind": kind, "rows": _log_int(rng, 1, 4096), "V": _log_int(rng, 2, 262144), "ld": rng.choice(("packed", "padded")),
                "dtype": rng.choice(tuple(DTYPES)), "T": rng.choice((1.0, 1.0, 0.7, round(rng.uniform(0.5, 2.0), 2)))}
        if rng.random() < 0.3:
            case["V"] = (case["V"] + 63) // 64 * 64
        case["padding"] = rng.choice((0, rng.randint(0, case["rows"] // 8)))
        if kind == "score":
            case["k"] = rng.choice((0, 0, 1, 5, 20, _log_int(rng, 1, 256)))
            case["rank"] = rng.random() < 0.5
        elif kind == "score_grad":
            case["entropy"] = rng.random() < 0.5
        else:
            case["bonus"] = rng.choice((0.0, 0.01, round(rng.uniform(0.001, 0.1), 3)))
        return case
    case = {"kind": kind, "P": _log_int(rng, 1, 32), "N": _log_int(rng, 100, 61000000), "ld": rng.choice(("packed", "padded", "padded")),
            "dtype": rng.choice(("fp32", "fp32", "bf16", "fp16"))}
    if kind == "norms":
        case["max_norm"] = rng.choice((0.5, 1.0, 5.0))
        return case
    case.update({"elastic": rng.random() < 0.5, "tensors": rng.choice((0, _log_int(rng, 1, 400))), "clip": rng.random() < 0.5,
                 "step": _log_int(rng, 1, 100000)})
    return case


def draw(rng):
    largest = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw_once(rng)
        if "rows" in case and (case["rows"] * case["V"] > 2048 * 131072 or case.get("k", 0) and case["rows"] * case["V"] > 512 * 131072):
            continue
        if "P" in case and case["P"] * case["N"] > 8 * 61000000:
            continue
        if work(case)["bytes"] <= largest:
            return case


# ---- inputs -------------------------------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _uniform(gen, shape, lo, hi):
    return torch.rand(shape, generator=gen, device="cuda") * (hi - lo) + lo


def _normal(gen, shape, std):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen)


def _logits(case, gen):
    """What a trained model puts out, a broad bulk and some candidates that stand out, and the tokens that were taken: mostly candidates."""
    rows, V = case["rows"], case["V"]
    ld = (V + 255) // 256 * 256 if case["ld"] == "padded" else V
    z = _normal(gen, (rows, ld), 2.0).to(DTYPES[case["dtype"]])[:, :V]
    peaks = min(V, 12)
    step = torch.randint(1, V // peaks + 1, (rows, 1), generator=gen, device="cuda")
    first = torch.randint(0, V, (rows, 1), generator=gen, device="cuda")
    places = (first + step * torch.arange(peaks, device="cuda")) % V
    z.scatter_(1, places, _uniform(gen, (rows, peaks), 4.0, 13.0).to(z.dtype))
    tokens = torch.gather(places, 1, torch.randint(0, peaks, (rows, 1), generator=gen, device="cuda")).squeeze(1)
    anywhere = torch.randint(0, V, (rows,), generator=gen, device="cuda")
    tokens = torch.where(torch.rand((rows,), generator=gen, device="cuda") < 0.2, anywhere, tokens).to(torch.int32)
    tokens[torch.randperm(rows, generator=gen, device="cuda")[:case["padding"]]] = -1
    return z, tokens


def _rows_state(case, gen):
    rows, V, kind = case["rows"], case["V"], case["kind"]
    z, tokens = _logits(case, gen)
    state = {"logits": z, "tokens": tokens}
    per_row = lambda dtype=torch.float32: torch.empty((rows,), dtype=dtype, device="cuda")
    like = lambda: torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device="cuda")
    if kind == "score":
        state["out"] = {"logprob": per_row(), "entropy": per_row()}
        if case["rank"]:
            state["out"]["rank"] = per_row(torch.int32)
        if case["k"]:
            state["out"]["top_logprob"] = torch.empty((rows, case["k"]), dtype=torch.float32, device="cuda")
            state["out"]["top_indices"] = torch.empty((rows, case["k"]), dtype=torch.int32, device="cuda")
    elif kind == "score_grad":
        # what the forward pass left behind: the rows' maxima, sums and entropies
        m, s, entropy = _statistics(z.float(), case["T"])
        live = (tokens >= 0).float()
        state["state"] = torch.stack((m * live, s * live, entropy * live, torch.zeros_like(m)), dim=1)
        state["dlogprob"] = _normal(gen, (rows,), 1.0) / rows
        state["dentropy"] = _uniform(gen, (rows,), 0.5, 1.5) * (0.01 / rows) if case["entropy"] else None
        state["out"] = {"dlogits": like()}
    else:
        state["weight"] = _normal(gen, (rows,), 1.0)                     # advantages: of either sign
        state["out"] = {"loss": per_row(), "logprob": per_row(), "dlogits": like()}
        if case["bonus"]:
            state["out"]["entropy"] = per_row()
    return state


def _ld(case):
    return (case["N"] + 255) // 256 * 256 if case["ld"] == "padded" else case["N"]


def _replicas(case, gen, std):
    return _normal(gen, (case["P"], _ld(case)), std)


def _gradients(case, gen):
    """Gradients whose size changes from one stretch of parameters to the next, as it does between layers."""
    g = _replicas(case, gen, 1e-3)
    stretch = max(1, case["N"] // 7)
    g *= torch.exp(_normal(gen, ((g.shape[1] + stretch - 1) // stretch,), 1.0)).repeat_interleave(stretch)[:g.shape[1]]
    return g


def _ends(case, gen):
    """Where the tensors of a replica end: a matrix and a vector in turn, of sizes that differ; the vectors are not decayed."""
    n, N = case["tensors"], case["N"]
    size = torch.exp(_normal(gen, (n,), 1.0)).double()
    size[1::2] *= 0.01
    ends = (size.cumsum(0) / size.sum() * N).round().to(torch.int64)
    ends[-1] = N
    rates = _uniform(gen, (n,), 0.5, 1.0)
    decays = torch.full((n,), 0.01, device="cuda")
    decays[1::2] = 0.0
    return ends, rates, decays


def _replica_state(case, gen):
    P, N, kind = case["P"], case["N"], case["kind"]
    g = _gradients(case, gen)
    state = {"G": g.to(DTYPES[case["dtype"]]), "P": P, "N": N}
    if kind == "norms":
        state["out"] = {"norm": torch.empty((P,), dtype=torch.float32, device="cuda"), "clip": torch.empty((P,), dtype=torch.float32, device="cuda")}
        return state
    ld = g.shape[1]
    state["W"] = _replicas(case, gen, 0.05)
    m = _replicas(case, gen, 1.0).mul_(g.abs()).mul_(0.4)
    v = _replicas(case, gen, 1.0).square_().mul_(g.square()).mul_(0.5).add_(1e-12)
    del g
    if kind == "adamw8":
        for name, moment, coder in (("M", m, _encode_m), ("S", v, _encode_s)):
            moment[:, N:] = 0.0
            code, state[name + "_scale"] = coder(_blocks(moment[:, :N]), torch.full((P, 1, 1), 1 << 15, device="cuda"))
            state[name] = torch.zeros((P, ld), dtype=torch.uint8, device="cuda")
            state[name][:, :N] = code.view(P, -1)[:, :N]
            state[name] = state[name].view(torch.float8_e4m3fn if name == "M" else torch.float8_e5m2)
    else:
        state["M"], state["S"] = m, v
    state["Wc"] = state["W"][:, :N].mean(dim=0) if case["elastic"] else None
    state["tensors"] = _ends(case, gen) if case["tensors"] else None
    state["clip"] = None
    if case["clip"]:
        state["clip"] = _uniform(gen, (P,), 0.0, 2.0).clamp(0.2, 1.0)    # most replicas' gradients are clipped, or none is
        if P >= 8:
            state["clip"][P // 2] = 0.0                                  # one diverged and sits this step out
    state["rule"] = {"eta": 2e-3, "rho": 0.1 if case["elastic"] else 0.0, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "decay": 0.01}
    return state


def prepare(case, seed):
    gen = _generator(seed)
    state = _rows_state(case, gen) if "rows" in case else _replica_state(case, gen)
    state["case"], state["seed"] = case, seed & 0x7fffffff
    return state


# ---- the plain form: rows of logits ---------------------------------------------------------------------------------

def _statistics(x, T):
    """Of every row: its maximum, the sum of exp((z - m)/T), the entropy of the softmax of z/T."""
    m = x.amax(dim=1, keepdim=True)
    y = (x - m) / T
    e = y.exp()
    s = e.sum(dim=1)
    entropy = s.log() - torch.where(e > 0, e * y, 0.0).sum(dim=1) / s
    return m.squeeze(1), s, entropy


def _first(x, k):
    """The k first of every row's order, ties to the lowest index: places are ranked by one whole number of the logit's order and the index."""
    V = x.shape[1]
    bits = (x + 0.0).view(torch.int32)                                   # -0 and 0 are one value
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    order = (order << 32) | (V - 1 - torch.arange(V, device=x.device))
    return V - 1 - (torch.topk(order, min(k, V), dim=1).values & 0xFFFFFFFF)


def _score(case, z, tokens):
    x = z.float()
    rows, V = x.shape
    m, s, entropy = _statistics(x, case["T"])
    live = tokens >= 0
    at = tokens.clamp(min=0).long().view(-1, 1)
    of_token = torch.gather(x, 1, at)
    log_s = s.log()
    out = {"logprob": torch.where(live, (of_token.squeeze(1) - m) / case["T"] - log_s, 0.0), "entropy": torch.where(live, entropy, 0.0)}
    if case["rank"]:
        before = (x > of_token) | ((x == of_token) & (torch.arange(V, device=x.device) < at))
        out["rank"] = torch.where(live, before.sum(dim=1), -1).to(torch.int32)
    if case["k"]:
        places = _first(x, case["k"])
        found = torch.gather(x, 1, places)
        there = (found > NEG) & live.view(-1, 1)
        values = torch.full((rows, case["k"]), NEG, device=x.device)
        indices = torch.full((rows, case["k"]), -1, dtype=torch.int32, device=x.device)
        values[:, :places.shape[1]] = torch.where(there, (found - m.view(-1, 1)) / case["T"] - log_s.view(-1, 1), NEG)
        indices[:, :places.shape[1]] = torch.where(there, places, -1).to(torch.int32)
        out["top_logprob"], out["top_indices"] = values, indices
    return out


def _slope(z, tokens, T, m, s, entropy, up_logprob, up_entropy):
    """The gradient of up_logprob * logprob + up_entropy * entropy."""
    y = (z.float() - m.view(-1, 1)) / T
    q = y.exp() / s.view(-1, 1)
    d = q * -up_logprob.view(-1, 1)
    d.scatter_add_(1, tokens.clamp(min=0).long().view(-1, 1), up_logprob.view(-1, 1).expand(-1, 1))
    if up_entropy is not None:
        log_q = y - s.log().view(-1, 1)
        d -= torch.where(q > 0, q * (log_q + entropy.view(-1, 1)), 0.0) * up_entropy.view(-1, 1)
    return torch.where((tokens >= 0).view(-1, 1), d / T, 0.0).to(z.dtype)


def _score_grad(case, state):
    m, s, entropy, _ = state["state"].unbind(dim=1)
    return {"dlogits": _slope(state["logits"], state["tokens"], case["T"], m, s, entropy, state["dlogprob"], state["dentropy"])}


def _token_loss(case, state):
    z, tokens = state["logits"], state["tokens"]
    rows = z.shape[0]
    x = z.float()
    m, s, entropy = _statistics(x, case["T"])
    live = tokens >= 0
    logprob = (torch.gather(x, 1, tokens.clamp(min=0).long().view(-1, 1)).squeeze(1) - m) / case["T"] - s.log()
    loss = -state["weight"] * logprob
    up_entropy = None
    if case["bonus"]:
        loss = loss - case["bonus"] * entropy
        up_entropy = torch.full_like(m, -case["bonus"] / rows)
    out = {"loss": torch.where(live, loss, 0.0), "logprob": torch.where(live, logprob, 0.0),
           "dlogits": _slope(z, tokens, case["T"], m, s, entropy, state["weight"] * (-1.0 / rows), up_entropy)}
    if case["bonus"]:
        out["entropy"] = torch.where(live, entropy, 0.0)
    return out


# ---- the plain form: replicas ---------------------------------------------------------------------------------------

def _norms(case, state):
    g = state["G"][:, :state["N"]]
    norm = (g.float().square().sum(dim=1) if g.dtype != torch.float32 else g.square().sum(dim=1)).sqrt()
    limit = torch.full_like(norm, case["max_norm"])
    clip = torch.where(norm <= limit, 1.0, limit / norm)
    return {"norm": norm, "clip": torch.where(norm.isfinite(), clip, 0.0)}


def _blocks(x):
    """[P][N] as [P][blocks][256], zeros behind the end."""
    P, N = x.shape
    return torch.nn.functional.pad(x, (0, -N % BLOCK)).view(P, -1, BLOCK)


def _mix(x):
    """A whole number of 32 bits for another, every bit of it depending on all of x's."""
    x = (x ^ (x >> 16)) * 0x6C8E9CF5 & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x2F5D7A4B & 0xFFFFFFFF
    return x ^ (x >> 16)


def _dither(P, N, step, seed, device):
    """16 random bits for every parameter of every worker, from its number, the worker's, the step's and the seed alone."""
    worker = torch.arange(P, device=device, dtype=torch.int64).view(P, 1, 1)
    word = torch.arange(2, device=device, dtype=torch.int64)
    key = _mix((_mix((seed + worker * 0x9E3779B1) & 0xFFFFFFFF) + step * 0x85157AF5 + word * 0x632BE5AB) & 0xFFFFFFFF)
    group = torch.arange((N + BLOCK - 1) // BLOCK * (BLOCK // 4), device=device, dtype=torch.int64).view(1, -1, 1)
    h = _mix(group ^ key).view(P, -1, 2, 1)
    return (h >> torch.tensor((0, 16), device=device)).bitwise_and_(0xFFFF).to(torch.int32).view(P, -1, BLOCK)


def _encode(x, bits, top, dither):
    """Blocks of numbers from 0 on in 8 bits with `bits` of fraction, rounded up or down at random, and their powers of two."""
    most = x.view(torch.int32).amax(dim=2, keepdim=True)
    there = most < 0x7F800000                                            # neither infinite nor NaN
    scale = ((most >> 23) - top).clamp_(min=1)
    inverse = ((254 - scale) << 23).view(torch.float32)
    unit = 2.0 ** (-112 if bits == 2 else -120)                          # the type's smallest exponent meets that of 32 bits
    code = (x * inverse * unit).view(torch.int32)
    code = (code + (dither << (7 - bits)) + (1 << (6 - bits))) >> (23 - bits)
    code = torch.where(there, code, 0).to(torch.uint8)
    return code, torch.where(there, (scale << 23).view(torch.float32), float("nan")).squeeze(2)


def _encode_m(x, dither):
    code, scale = _encode(x.abs(), 3, 7, dither)
    return code | ((x < 0).to(torch.uint8) << 7), scale


def _encode_s(x, dither):
    code, scale = _encode(x, 2, 14, dither)
    return torch.maximum(code, (x > 0).to(torch.uint8)), scale           # what is above 0 stays above 0


def _decode(code, scale, N):
    P = code.shape[0]
    return _blocks(code[:, :N].float()).mul_(scale.unsqueeze(2)).view(P, -1)[:, :N]


def _single(x):
    """A number as 32 bits hold it."""
    return torch.tensor(x, dtype=torch.float32).item()


def _adamw(case, state):
    W, N, rule, step = state["W"][:, :state["N"]], state["N"], state["rule"], case["step"]
    beta1, beta2 = _single(rule["beta1"]), _single(rule["beta2"])
    eight = case["kind"] == "adamw8"
    g = state["G"][:, :N].float()
    live = None
    if state["clip"] is not None:
        g = g * state["clip"].view(-1, 1)
        live = (state["clip"] != 0.0).view(-1, 1)
    m_old = _decode(state["M"], state["M_scale"], N) if eight else state["M"][:, :N]
    v_old = _decode(state["S"], state["S_scale"], N) if eight else state["S"][:, :N]
    m = m_old * beta1 + g * (1.0 - beta1)
    v = v_old * beta2 + (g * (1.0 - beta2)) * g
    del g, m_old, v_old
    eta, decay = rule["eta"], rule["decay"]
    if state["tensors"] is not None:
        ends, rates, decays = state["tensors"]
        length = torch.diff(ends, prepend=ends.new_zeros(1))
        eta = eta * torch.repeat_interleave(rates, length, output_size=N)
        decay = torch.repeat_interleave(decays, length, output_size=N)
    d = v.sqrt().mul_(1.0 / math.sqrt(1.0 - beta2 ** step)).add_(rule["eps"])
    d = torch.div(m, d, out=d).mul_(1.0 / (1.0 - beta1 ** step)).add_(W * decay).mul_(eta)
    if live is not None:
        d = torch.where(live, d, 0.0)
    out = {"W": W}
    if state["Wc"] is not None:
        alpha = rule["eta"] * rule["rho"]
        apart = W - state["Wc"]
        d.add_(apart, alpha=alpha)
        state["Wc"].add_(apart.sum(dim=0), alpha=alpha)
        del apart
        out["Wc"] = state["Wc"]
    W.sub_(d)
    del d
    if not eight:
        for name, moment in (("M", m), ("S", v)):
            out[name] = state[name][:, :N]
            out[name].copy_(moment if live is None else torch.where(live, moment, out[name]))
        return out
    dither = _dither(case["P"], N, step, state["seed"], W.device)
    for name, moment, coder in (("M", m, _encode_m), ("S", v, _encode_s)):
        code, scale = coder(_blocks(moment), dither)
        code = code.view(case["P"], -1)[:, :N]
        held, held_scale = state[name].view(torch.uint8)[:, :N], state[name + "_scale"]
        held.copy_(code if live is None else torch.where(live, code, held))
        held_scale.copy_(scale if live is None else torch.where(live, scale, held_scale))
        out[name], out[name + "_scale"] = state[name][:, :N], held_scale
    return out


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["kind"] == "score":
        return _score(case, state["logits"], state["tokens"])
    if case["kind"] == "score_grad":
        return _score_grad(case, state)
    if case["kind"] == "token_loss":
        return _token_loss(case, state)
    return _norms(case, state) if case["kind"] == "norms" else _adamw(case, state)


# ---- the framework's calls ------------------------------------------------------------------------------------------

def _own(state):
    import paper_1708_02983_amd as hip
    case, kind = state["case"], state["case"]["kind"]
    if "rows" in case:
        z, tokens, T, out = state["logits"], state["tokens"], case["T"], state["out"]
        if kind == "score":
            hip.easgd_score_tokens(z, tokens, temperature=T, k=case["k"], **out)
        elif kind == "score_grad":
            hip.easgd_score_tokens_grad(z, tokens, state["state"], temperature=T, dlogprob=state["dlogprob"], dentropy=state["dentropy"], **out)
        else:
            hip.easgd_token_loss(z, tokens, weight=state["weight"], bonus=case["bonus"], temperature=T, scale=1.0 / case["rows"], **out)
        return out
    if kind == "norms":
        hip.easgd_grad_norms(state["G"], max_norm=case["max_norm"], N=state["N"], **state["out"])
        return state["out"]
    N = state["N"]
    names = ["M", "S"]
    eight = {}
    if kind == "adamw8":
        eight = {"M_scale": state["M_scale"], "S_scale": state["S_scale"], "seed": state["seed"]}
    hip.adamw_round(state["W"], state["M"], state["S"], state["G"], case["step"], Wc=state["Wc"], tensors=state["tensors"], clip=state["clip"], N=N,
                    **state["rule"], **eight)
    out = {"W": state["W"][:, :N]}
    if state["Wc"] is not None:
        out["Wc"] = state["Wc"]
    for name in names:
        out[name] = state[name][:, :N]
        if eight:
            out[name + "_scale"] = state[name + "_scale"]
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if "rows" in case:
        size = 4 if case["dtype"] == "fp32" else 2
        read = (case["rows"] - case["padding"]) * case["V"]              # padded rows are not looked at
        each = case["rows"] * case["V"]
        if kind == "score":
            return {"bytes": read * size + case["rows"] * (12 + 4 * case["rank"] + 8 * case["k"]), "flops": 5 * read}
        if kind == "score_grad":
            return {"bytes": (read + each) * size + case["rows"] * (24 + 4 * case["entropy"]), "flops": (6 if case["entropy"] else 4) * read}
        return {"bytes": (read + each) * size + case["rows"] * (16 + 4 * (case["bonus"] != 0.0)), "flops": (10 if case["bonus"] else 7) * read}
    each, size = case["P"] * case["N"], 4 if case["dtype"] == "fp32" else 2
    if kind == "norms":
        return {"bytes": each * size + 8 * case["P"], "flops": 2 * each}
    moments = 16 if kind == "adamw" else 4
    center = 8 * case["N"] if case["elastic"] else 0
    scales = 16 * case["P"] * ((case["N"] + BLOCK - 1) // BLOCK) if kind == "adamw8" else 0
    return {"bytes": each * (8 + size + moments) + center + scales + 16 * case["tensors"], "flops": (18 if case["elastic"] else 14) * each}


# ---- the same from the definitions in 64 bits -----------------------------------------------------------------------

def _exact_rows(case, state):
    T, rows = float(case["T"]), case["rows"]
    kind, parts = case["kind"], []
    step = max(1, (1 << 25) // case["V"])
    for at in range(0, rows, step):
        z = state["logits"][at:at + step].double()
        tokens = state["tokens"][at:at + step].long()
        padding = tokens < 0
        log_q = torch.log_softmax(z / T, dim=1)
        q = log_q.exp()
        entropy = -(q * log_q).nan_to_num(0.0).sum(dim=1)
        hot = torch.zeros_like(z)
        hot[torch.arange(len(tokens), device=z.device), tokens.clamp(min=0)] = 1.0
        logprob = (hot * log_q.clamp(min=-1e300)).sum(dim=1)
        part = {"logprob": logprob.masked_fill(padding, 0.0), "entropy": entropy.masked_fill(padding, 0.0)}
        if kind == "score":
            if case["k"]:
                first = torch.sort(log_q, dim=1, descending=True).values[:, :case["k"]]
                first = torch.nn.functional.pad(first, (0, case["k"] - first.shape[1]), value=NEG)
                part["top_logprob"] = first.masked_fill(padding.view(-1, 1), NEG)
        else:
            if kind == "score_grad":
                up, up_h = state["dlogprob"][at:at + step].double(), state["dentropy"]
                up_h = None if up_h is None else up_h[at:at + step].double()
            else:
                weight = state["weight"][at:at + step].double()
                part["loss"] = (-weight * logprob - case["bonus"] * entropy).masked_fill(padding, 0.0)
                up, up_h = -weight / rows, torch.full_like(weight, -case["bonus"] / rows)
            d = (hot - q) * up.view(-1, 1)
            if up_h is not None:
                d -= (q * (log_q + entropy.view(-1, 1))).nan_to_num(0.0) * up_h.view(-1, 1)
            part["dlogits"] = (d / T).masked_fill(padding.view(-1, 1), 0.0)
        parts.append(part)
    whole = {name: torch.cat([p[name] for p in parts]) for name in parts[0]}
    if kind == "score":
        if case["rank"]:
            whole["rank"] = None
        if case["k"]:
            whole["top_indices"] = None
        return whole
    names = ("dlogits",) if kind == "score_grad" else ("loss", "logprob", "dlogits", "entropy")
    return {name: whole[name] for name in names if name != "entropy" or case["bonus"]}


def _exact_adamw(case, state):
    N, P, rule, t = case["N"], case["P"], state["rule"], case["step"]
    b1, b2 = _single(rule["beta1"]), _single(rule["beta2"])
    eight = case["kind"] == "adamw8"
    eta = torch.full((N,), rule["eta"], dtype=torch.float64, device="cuda")
    decay = torch.full((N,), rule["decay"], dtype=torch.float64, device="cuda")
    if state["tensors"] is not None:
        which = torch.searchsorted(state["tensors"][0], torch.arange(N, device="cuda"), right=True)
        eta *= state["tensors"][1].double()[which]
        decay = state["tensors"][2].double()[which]
    center = None if state["Wc"] is None else state["Wc"].double()
    drift = torch.zeros((N,), dtype=torch.float64, device="cuda")
    out = {"W": torch.empty((P, N), dtype=torch.float64, device="cuda")}
    if not eight:
        out["M"], out["S"] = torch.empty_like(out["W"]), torch.empty_like(out["W"])
    for i in range(P):
        w, m, v = (state[name][i, :N].float().double() for name in ("W", "M", "S"))
        if eight:
            m *= state["M_scale"][i].double().repeat_interleave(BLOCK)[:N]
            v *= state["S_scale"][i].double().repeat_interleave(BLOCK)[:N]
        clip = 1.0 if state["clip"] is None else state["clip"][i].item()
        moved = torch.zeros_like(w)
        if clip != 0.0:
            g = clip * state["G"][i, :N].double()
            m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
            moved = eta * (m / (1 - b1 ** t) / ((v / (1 - b2 ** t)).sqrt() + rule["eps"]) + decay * w)
        if center is not None:
            drift += w - center
            moved += rule["eta"] * rule["rho"] * (w - center)
        out["W"][i] = w - moved
        if not eight:
            out["M"][i], out["S"][i] = m, v
    if center is not None:
        out["Wc"] = center + rule["eta"] * rule["rho"] * drift
    if eight:
        for name in ("M", "S"):
            out[name], out[name + "_scale"] = None, None                 # rounded at random: no one value
    order = ["W"] + (["Wc"] if center is not None else []) + (["M", "M_scale", "S", "S_scale"] if eight else ["M", "S"])
    return {name: out[name] for name in order}


def exact(case, seed):
    state = prepare(case, seed)
    if "rows" in case:
        return _exact_rows(case, state)
    if case["kind"] == "norms":
        norm = torch.stack([g.double().square().sum().sqrt() for g in state["G"][:, :case["N"]]])
        return {"norm": norm, "clip": (case["max_norm"] / norm).clamp(max=1.0)}
    return _exact_adamw(case, state)
