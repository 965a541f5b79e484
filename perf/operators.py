"""The operators on rows of logits that are timed, and the ranges that they stand for.

  * ``easgd_top_logits``: the k largest logits of every row with their indices, and the row's log-sum-exp: what a teacher
    hands on (kind "top");
  * ``easgd_distill``, ``easgd_distill_loss``, ``easgd_distill_grad``: the loss of a student against a teacher's top
    logits, mixed with the cross-entropy of a label, and its gradient: in one call, forward only, backward only
    (kinds "distill", "distill_loss", "distill_grad");
  * ``easgd_sample_tokens``: one token a row with temperature, top-k, top-p and min-p from given random numbers
    (kind "sample").

With ``own`` false ``run`` computes the same from elementary torch operations.  ``rows`` counts rows of logits, ``V`` is
their length, ``ld`` ("packed" or "padded" to a multiple of 256) how far they lie apart.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
NEG = float("-inf")


def listed():
    return [
        # a teacher scores a batch of positions of a large vocabulary: the largest read
        {"name": "teacher_top_batch", "kind": "top", "rows": 2048, "V": 131072, "ld": "packed", "dtype": "bf16", "k": 64, "T": 2.0},
        # the teacher beside a student that answers token by token: a few rows of an odd vocabulary, every row at another alignment
        {"name": "teacher_top_decode", "kind": "top", "rows": 8, "V": 50001, "ld": "packed", "dtype": "fp16", "k": 20, "T": 1.0},
        # the center as the teacher of sixteen workers of 128 samples each, a thousand classes
        {"name": "center_top_classes", "kind": "top", "rows": 2048, "V": 1000, "ld": "packed", "dtype": "fp32", "k": 10, "T": 4.0},
        # the training step of the large vocabulary: loss and gradient, labels mixed in, padded positions
        {"name": "distill_batch", "kind": "distill", "rows": 2048, "V": 131072, "ld": "packed", "dtype": "bf16", "k": 64, "T": 2.0,
         "tail": False, "hard": 0.5, "padding": 128},
        # an odd vocabulary and number of rows, the teacher's rest as one more outcome
        {"name": "distill_odd_tail", "kind": "distill", "rows": 777, "V": 50001, "ld": "packed", "dtype": "fp16", "k": 33, "T": 1.0,
         "tail": True, "hard": 0.0, "padding": 0},
        # the framework's own networks: sixteen workers, 128 samples, a hundred classes: launches and latency
        {"name": "distill_classes", "kind": "distill", "rows": 2048, "V": 100, "ld": "packed", "dtype": "fp32", "k": 10, "T": 4.0,
         "tail": False, "hard": 0.1, "padding": 0},
        # backward alone, for a program that differentiates what it did with the losses
        {"name": "distill_backward", "kind": "distill_grad", "rows": 1024, "V": 32000, "ld": "padded", "dtype": "bf16", "k": 128, "T": 1.5,
         "tail": True, "hard": 0.25, "padding": 64},
        # forward alone on a few very long rows: an evaluation in 32 bits
        {"name": "distill_forward_long", "kind": "distill_loss", "rows": 16, "V": 262144, "ld": "packed", "dtype": "fp32", "k": 256, "T": 1.0,
         "tail": True, "hard": 0.0, "padding": 0},
        # one conversation: latency
        {"name": "sample_one", "kind": "sample", "rows": 1, "V": 131072, "ld": "packed", "dtype": "bf16", "filters": "chat"},
        # a server's batch whose requests ask for different things, greedy ones and constrained ones among them
        {"name": "sample_batch", "kind": "sample", "rows": 256, "V": 131072, "ld": "packed", "dtype": "bf16", "filters": "mixed"},
        # nucleus sampling in 32 bits of an odd vocabulary
        {"name": "sample_nucleus", "kind": "sample", "rows": 64, "V": 50001, "ld": "packed", "dtype": "fp32", "filters": "nucleus"},
        # answers for training: the whole distribution, no filter
        {"name": "sample_whole", "kind": "sample", "rows": 512, "V": 32000, "ld": "padded", "dtype": "fp16", "filters": "none"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    kind = rng.choice(("top", "distill", "distill", "distill_loss", "distill_grad", "sample", "sample"))
    case = {"kind": kind, "rows": _log_int(rng, 1, 4096), "V": _log_int(rng, 2, 262144), "ld": rng.choice(("packed", "padded")),
            "dtype": rng.choice(tuple(DTYPES))}
    if rng.random() < 0.3:
        case["V"] = (case["V"] + 63) // 64 * 64
    if kind == "sample":
        case["filters"] = rng.choice(("chat", "mixed", "mixed", "nucleus", "none"))
        return case
    case["k"] = _log_int(rng, 1, 256)
    case["T"] = rng.choice((1.0, 1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)))
    if kind != "top":
        case["tail"] = rng.random() < 0.5
        case["hard"] = rng.choice((0.0, 0.5, round(rng.uniform(0.05, 1.0), 2)))
        case["padding"] = 0 if case["hard"] == 0.0 else rng.randint(0, case["rows"] // 8)
    return case


def draw(rng):
    largest = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw_once(rng)
        # sampling sorts whole rows in its plain form: no more logits than the largest listed batch
        if case["kind"] == "sample" and case["rows"] * case["V"] > 256 * 131072:
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


def _places(gen, rows, V, n):
    """n distinct places in every row."""
    step = torch.randint(1, V // n + 1, (rows, 1), generator=gen, device="cuda")
    first = torch.randint(0, V, (rows, 1), generator=gen, device="cuda")
    return (first + step * torch.arange(n, device="cuda")) % V


def _logits(case, gen):
    """What a trained model puts out: a broad bulk, and a few candidates that stand out in every row."""
    rows, V = case["rows"], case["V"]
    ld = (V + 255) // 256 * 256 if case["ld"] == "padded" else V
    z = torch.empty((rows, ld), dtype=torch.float32, device="cuda").normal_(0.0, 2.0, generator=gen)
    z = z.to(DTYPES[case["dtype"]])[:, :V]
    peaks = min(V, 12)
    z.scatter_(1, _places(gen, rows, V, peaks), _uniform(gen, (rows, peaks), 4.0, 13.0).to(z.dtype))
    return z


def _teacher(case, gen, z):
    """A teacher's top logits for these rows: distinct places, logits in descending order, the student near them."""
    rows, V, k = case["rows"], case["V"], case["k"]
    live = min(k, V)
    places = _places(gen, rows, V, live)
    logits = (_uniform(gen, (rows, live), 0.0, 1.0).pow(3) * 10.0 + 2.0).sort(dim=1, descending=True).values
    z.scatter_(1, places, (logits + _uniform(gen, (rows, live), -1.5, 1.5)).to(z.dtype))
    indices = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
    values = torch.full((rows, k), NEG, dtype=torch.float32, device="cuda")
    indices[:, :live] = places.to(torch.int32)
    values[:, :live] = logits
    lse = torch.logsumexp(logits / case["T"], dim=1) + _uniform(gen, (rows,), 0.02, 0.3)
    return indices, values, lse


def _filters(case, gen):
    """Temperature, top-k, top-p and min-p of every row; None where nobody asks for one."""
    rows, kind = case["rows"], case["filters"]
    if kind == "none":
        return _uniform(gen, (rows,), 0.8, 1.2), None, None, None
    if kind == "nucleus":
        return _uniform(gen, (rows,), 0.7, 1.1), None, _uniform(gen, (rows,), 0.85, 0.97), None
    if kind == "chat":
        return (_uniform(gen, (rows,), 0.6, 0.8), torch.full((rows,), 50, dtype=torch.int32, device="cuda"),
                torch.full((rows,), 0.9, device="cuda"), torch.full((rows,), 0.02, device="cuda"))
    pick = torch.randint(0, 8, (4, rows), generator=gen, device="cuda")
    temperature = _uniform(gen, (rows,), 0.5, 1.3)
    temperature[pick[0] == 0] = 0.0                                       # greedy
    top_k = torch.randint(1, 200, (rows,), generator=gen, device="cuda").to(torch.int32)
    top_k[pick[1] < 3] = 0                                                # none
    top_p = _uniform(gen, (rows,), 0.5, 0.99)
    top_p[pick[2] < 2] = 1.0                                              # none
    min_p = _uniform(gen, (rows,), 0.01, 0.2)
    min_p[pick[3] < 4] = 0.0                                              # none
    return temperature, top_k, top_p, min_p


def _inputs(case, seed):
    gen = _generator(seed)
    z = _logits(case, gen)
    rows, V = case["rows"], case["V"]
    got = {"logits": z}
    if case["kind"] == "sample":
        if case["filters"] == "mixed":                                    # every eighth row may answer with a few tokens only
            allowed = torch.zeros((rows, V), dtype=torch.bool, device="cuda")
            allowed.scatter_(1, torch.randint(0, V, (rows, min(V, 40)), generator=gen, device="cuda"), True)
            allowed |= (torch.arange(rows, device="cuda") % 8 != 3).view(-1, 1)
            z.masked_fill_(~allowed, NEG)
        got["temperature"], got["top_k"], got["top_p"], got["min_p"] = _filters(case, gen)
        got["u"] = torch.rand((rows,), generator=gen, device="cuda")
        return got
    if case["kind"] == "top":
        return got
    got["indices"], got["values"], lse = _teacher(case, gen, z)
    got["teacher_lse"] = lse if case["tail"] else None
    got["labels"] = None
    if case["hard"] > 0.0:
        labels = torch.randint(0, V, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        labels[torch.randperm(rows, generator=gen, device="cuda")[:case["padding"]]] = -1
        got["labels"] = labels
    if case["kind"] == "distill_grad":
        got["dloss"] = _uniform(gen, (rows,), 0.5, 1.5) / rows
    return got


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    rows = case["rows"]
    z = state["logits"]
    if case["kind"] == "top":
        state["out"] = {"values": torch.empty((rows, case["k"]), dtype=torch.float32, device="cuda"),
                        "indices": torch.empty((rows, case["k"]), dtype=torch.int32, device="cuda"),
                        "lse": torch.empty((rows,), dtype=torch.float32, device="cuda")}
    elif case["kind"] == "sample":
        state["out"] = {"tokens": torch.empty((rows,), dtype=torch.int32, device="cuda"),
                        "logprob": torch.empty((rows,), dtype=torch.float32, device="cuda")}
    else:
        state["out"] = {"loss": torch.empty((rows,), dtype=torch.float32, device="cuda"), "dlogits": torch.empty_strided(z.shape, z.stride(), dtype=z.dtype, device="cuda")}
    if case["kind"] == "distill_grad":
        # what the forward pass left behind for this backward pass: the rows' maxima and sums
        state["state"] = _statistics(case, state)
    return state


# ---- the plain form -----------------------------------------------------------------------------------------------

def _top(case, z):
    """Ties go to the lowest index: places are ranked by one whole number that holds the logit's order and the index."""
    V = z.shape[1]
    x = z.float() + 0.0                                                   # -0 and 0 are one value
    bits = x.view(torch.int32)
    order = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF).long()
    order = (order << 32) | (V - 1 - torch.arange(V, device=z.device))
    best = torch.topk(order, min(case["k"], V), dim=1).values
    places = V - 1 - (best & 0xFFFFFFFF)
    found = torch.gather(x, 1, places)
    values = torch.full((z.shape[0], case["k"]), NEG, dtype=torch.float32, device=z.device)
    indices = torch.full((z.shape[0], case["k"]), -1, dtype=torch.int32, device=z.device)
    values[:, :places.shape[1]] = found
    indices[:, :places.shape[1]] = torch.where(found > NEG, places, -1).to(torch.int32)
    m = x.amax(dim=1, keepdim=True)
    lse = m.squeeze(1) / case["T"] + ((x - m) / case["T"]).exp().sum(dim=1).log()
    return {"values": values, "indices": indices, "lse": lse}


def _soft(case, given):
    """The teacher's probabilities of its places in 64 bits (what is left over comes from a difference), and what is left over."""
    used = given["indices"] >= 0
    a = given["values"].double() / case["T"]
    if given["teacher_lse"] is None:
        p = torch.softmax(a, dim=1)
        return used, p, None
    p = torch.where(used, (a - given["teacher_lse"].double().view(-1, 1)).exp(), 0.0)
    return used, p, (1.0 - p.sum(dim=1)).clamp(min=0.0)


def _statistics(case, given):
    """Of every row: its maximum m, the sums of exp((z - m)/T) and exp(z - m), and the first sum's part outside the teacher's places."""
    z = given["logits"].float()
    m = z.amax(dim=1, keepdim=True)
    e = ((z - m) / case["T"]).exp()
    total = e.sum(dim=1)
    hard = (z - m).exp().sum(dim=1)
    outside = torch.zeros_like(total)
    if given["teacher_lse"] is not None:
        # a slot that is not used shares its row's first place, which is always a used one
        places = torch.where(given["indices"] >= 0, given["indices"], given["indices"][:, :1]).long()
        outside = e.scatter_(1, places, 0.0).sum(dim=1)
    return torch.stack((m.squeeze(1), total, hard, outside), dim=1)


def _loss(case, given, stats):
    z = given["logits"]
    used, p, rest = _soft(case, given)
    m, total, hard, outside = (s.double() for s in stats.unbind(dim=1))
    q = (torch.gather(z, 1, given["indices"].clamp(min=0).long()).double() - m.view(-1, 1)) / case["T"] - total.log().view(-1, 1)
    kl = torch.where(p > 0, p * (p.log() - q), 0.0).sum(dim=1)
    if rest is not None:
        kl = kl + torch.where((rest > 0) & (outside > 0), rest * (rest.log() - outside.log() + total.log()), 0.0)
    loss = (1.0 - case["hard"]) * case["T"] ** 2 * kl
    if given["labels"] is None:
        return loss.float()
    label = given["labels"].long()
    ce = m + hard.log() - torch.gather(z, 1, label.clamp(min=0).view(-1, 1)).squeeze(1).double()
    return torch.where(label >= 0, loss + case["hard"] * ce, 0.0).float()


def _gradient(case, given, stats, upstream):
    z = given["logits"].float()
    used, p, rest = _soft(case, given)
    m, total, hard, outside = (s.view(-1, 1) for s in stats.unbind(dim=1))
    q = ((z - m) / case["T"]).exp() / total
    if rest is None:
        soft = q.scatter_add(1, given["indices"].clamp(min=0).long(), torch.where(used, -p, 0.0).float())
    else:
        # without any place outside, the outcome "another place" is left out, and the probabilities sum up to what there is
        rest = torch.where(outside > 0, rest.view(-1, 1), 0.0)
        mass = p.sum(dim=1, keepdim=True) + rest
        factor = mass - rest * total.double() / outside.double().clamp(min=1e-300)
        places = torch.where(used, given["indices"], given["indices"][:, :1]).long()
        at = torch.gather(q, 1, places) * mass.float() - torch.where(used, p, p[:, :1]).float()
        soft = (q * factor.float()).scatter(1, places, at)
    d = soft * ((1.0 - case["hard"]) * case["T"])
    if given["labels"] is not None:
        label = given["labels"].long().view(-1, 1)
        ce = (z - m).exp() / hard
        ce.scatter_add_(1, label.clamp(min=0), torch.full_like(ce[:, :1], -1.0))
        d = torch.where(label >= 0, d + ce * case["hard"], 0.0)
    return (d * upstream).to(given["logits"].dtype)


def _sample(given):
    z = given["logits"].double()
    rows, V = z.shape
    temperature = given["temperature"].double().view(-1, 1)
    best, order = torch.sort(given["logits"], dim=1, descending=True, stable=True)
    m = z.amax(dim=1, keepdim=True)
    w = torch.where(z == m, 1.0, ((z - m) / temperature.clamp(min=1e-300)).exp())
    ranked = torch.gather(w, 1, order)
    place = torch.arange(V, device=z.device).view(1, -1)
    keep = (best > NEG).expand(rows, V).clone()
    keep &= (temperature > 0) | (place == 0)
    if given["top_k"] is not None:
        top_k = given["top_k"].long().view(-1, 1)
        keep &= (place < top_k) | (top_k <= 0)
    within = torch.where(keep, ranked, 0.0)
    if given["top_p"] is not None:
        top_p = given["top_p"].double().view(-1, 1)
        before = within.cumsum(dim=1) - within
        keep &= (before < top_p * within.sum(dim=1, keepdim=True)) | (top_p >= 1.0) | (place == 0)
    if given["min_p"] is not None:
        keep &= (ranked >= given["min_p"].double().view(-1, 1)) | (place == 0)
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ranked, 0.0))
    running = kept.cumsum(dim=1)
    mass = running[:, -1:]
    passed = running > given["u"].double().view(-1, 1) * mass
    token = torch.where(passed, place, V).amin(dim=1)
    last = torch.where(kept > 0, place, -1).amax(dim=1)
    token = torch.minimum(token, last)
    logprob = (torch.gather(kept, 1, token.clamp(min=0).view(-1, 1)) / mass).log().squeeze(1)
    return {"tokens": token.to(torch.int32), "logprob": logprob.float()}


def run(state):
    if own:
        return _own(state)
    case = state["case"]
    if case["kind"] == "top":
        return _top(case, state["logits"])
    if case["kind"] == "sample":
        return _sample(state)
    if case["kind"] == "distill_grad":
        return {"dlogits": _gradient(case, state, state["state"], state["dloss"].view(-1, 1))}
    stats = _statistics(case, state)
    out = {"loss": _loss(case, state, stats)}
    if case["kind"] == "distill":
        out["dlogits"] = _gradient(case, state, stats, 1.0 / case["rows"])
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------

def _own(state):
    import paper_1708_02983_amd as hip
    case, out = state["case"], state["out"]
    if case["kind"] == "top":
        hip.easgd_top_logits(state["logits"], case["k"], temperature=case["T"], values=out["values"], indices=out["indices"], lse=out["lse"])
        return out
    if case["kind"] == "sample":
        hip.easgd_sample_tokens(state["logits"], state["u"], temperature=state["temperature"], top_k=state["top_k"], top_p=state["top_p"],
                                min_p=state["min_p"], tokens=out["tokens"], logprob=out["logprob"])
        return out
    teacher = {"temperature": case["T"], "teacher_lse": state["teacher_lse"], "labels": state["labels"], "hard": case["hard"]}
    if case["kind"] == "distill":
        hip.easgd_distill(state["logits"], state["indices"], state["values"], scale=1.0 / case["rows"], loss=out["loss"], dlogits=out["dlogits"], **teacher)
        return {"loss": out["loss"], "dlogits": out["dlogits"]}
    if case["kind"] == "distill_loss":
        hip.easgd_distill_loss(state["logits"], state["indices"], state["values"], loss=out["loss"], **teacher)
        return {"loss": out["loss"]}
    hip.easgd_distill_grad(state["logits"], state["indices"], state["values"], state["state"], dloss=state["dloss"], dlogits=out["dlogits"], **teacher)
    return {"dlogits": out["dlogits"]}


# ---- what a pass cannot do without --------------------------------------------------------------------------------

def work(case):
    rows, V = case["rows"], case["V"]
    size = 4 if case["dtype"] == "fp32" else 2
    logits = rows * V * size
    if case["kind"] == "top":
        return {"bytes": logits + rows * (8 * case["k"] + 4), "flops": 4 * rows * V}
    if case["kind"] == "sample":
        return {"bytes": logits + rows * 28, "flops": 4 * rows * V}
    live = (rows - case["padding"]) * V                                   # padded rows are written, not read
    teacher = rows * (8 * case["k"] + 12)
    if case["kind"] == "distill_loss":
        return {"bytes": live * size + teacher, "flops": 4 * live}
    return {"bytes": live * size + logits + teacher, "flops": 8 * live}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _exact_sample(given):
    """Row by row on the host, as the filters are defined: an order, three prefixes of it, a walk in index order."""
    import numpy as np
    host = {k: None if v is None else (v.double() if v.is_floating_point() else v).cpu().numpy() for k, v in given.items() if k != "case"}
    tokens, logprobs = [], []
    for i, z in enumerate(host["logits"]):
        order = np.argsort(-z, kind="stable")
        order = order[np.isfinite(z[order])]
        T = host["temperature"][i]
        n = len(order)
        if T <= 0.0:
            n = 1
        w = np.exp((z[order] - z[order[0]]) / (T if T > 0.0 else 1.0))
        if host["top_k"] is not None and host["top_k"][i] > 0:
            n = min(n, int(host["top_k"][i]))
        first = n
        if host["top_p"] is not None and host["top_p"][i] < 1.0:
            sums = np.cumsum(w[:first])
            n = min(n, int(np.searchsorted(sums, host["top_p"][i] * sums[-1], side="left")) + 1)
        if host["min_p"] is not None:
            n = min(n, max(1, int(np.count_nonzero(w[:first] >= host["min_p"][i]))))
        back = np.argsort(order[:n])
        places, kept = order[:n][back], w[:n][back]
        sums = np.cumsum(kept)
        at = min(int(np.searchsorted(sums, host["u"][i] * sums[-1], side="right")), n - 1)
        tokens.append(places[at])
        logprobs.append(np.log(kept[at] / sums[-1]))
    return {"tokens": torch.tensor(np.array(tokens), dtype=torch.int32), "logprob": torch.tensor(np.array(logprobs), dtype=torch.float64)}


def _exact_top(case, z):
    rows, V = z.shape
    k = case["k"]
    values = torch.full((rows, k), NEG, dtype=torch.float64)
    indices = torch.full((rows, k), -1, dtype=torch.int32)
    lse = torch.empty(rows, dtype=torch.float64)
    step = max(1, 33_000_000 // V)
    for at in range(0, rows, step):
        part = z[at:at + step].double()
        best, order = torch.sort(part, dim=1, descending=True, stable=True)
        n = min(k, V)
        values[at:at + step, :n] = best[:, :n].cpu()
        indices[at:at + step, :n] = torch.where(best[:, :n] > NEG, order[:, :n], -1).to(torch.int32).cpu()
        lse[at:at + step] = torch.logsumexp(part / case["T"], dim=1).cpu()
    return {"values": values, "indices": indices, "lse": lse}


def _exact_losses(case, z, given, at):
    """The losses of some rows of logits (64 bits) from probabilities over the places and one more for all others."""
    T, h = case["T"], case["hard"]
    n, V = z.shape
    rows = slice(at, at + n)
    indices = given["indices"][rows].long()
    a = given["values"][rows].double() / T
    lq = torch.log_softmax(z / T, dim=1)
    extended = torch.cat((lq, torch.zeros_like(lq[:, :1])), dim=1)        # a column for the slots that are not used
    at_places = torch.gather(extended, 1, torch.where(indices >= 0, indices, V))
    lp = a - torch.logsumexp(a, dim=1, keepdim=True) if given["teacher_lse"] is None else a - given["teacher_lse"][rows].double().view(-1, 1)
    lp = torch.where(indices >= 0, lp, 0.0)
    p = torch.where(indices >= 0, lp.exp(), 0.0)
    kl = (p * (lp - at_places)).sum(dim=1)
    if given["teacher_lse"] is not None:
        others = torch.ones_like(extended, dtype=torch.bool).scatter(1, torch.where(indices >= 0, indices, V), False)[:, :V]
        some = others.any(dim=1)
        rest = (1.0 - p.sum(dim=1)).clamp(min=0.0)
        log_outside = torch.logsumexp(lq.masked_fill(~others, NEG).masked_fill(~some.view(-1, 1), 0.0), dim=1)
        kl = kl + torch.where(some & (rest > 0), torch.xlogy(rest, rest) - rest * log_outside, 0.0)
    loss = (1.0 - h) * T * T * kl
    if given["labels"] is not None:
        label = given["labels"][rows].long()
        ce = torch.nn.functional.cross_entropy(z, label.clamp(min=0), reduction="none")
        loss = torch.where(label >= 0, loss + h * ce, torch.zeros_like(loss))
    return loss


def exact(case, seed):
    given = _inputs(case, seed)
    if case["kind"] == "sample":
        return _exact_sample(given)
    if case["kind"] == "top":
        return _exact_top(case, given["logits"])
    # the gradient of the 64-bit losses, by differentiation
    rows, V = given["logits"].shape
    wide = case["kind"] != "distill_loss"
    upstream = given["dloss"].double() if case["kind"] == "distill_grad" else torch.full((rows,), 1.0 / rows, dtype=torch.float64, device="cuda")
    losses, gradients = [], []
    step = max(1, 33_000_000 // V)
    for at in range(0, rows, step):
        z = given["logits"][at:at + step].double().requires_grad_(wide)
        part = _exact_losses(case, z, given, at)
        losses.append(part.detach())
        if wide:
            gradients.append(torch.autograd.grad((part * upstream[at:at + step]).sum(), z)[0])
    out = {} if case["kind"] == "distill_grad" else {"loss": torch.cat(losses)}
    if wide:
        out["dlogits"] = torch.cat(gradients)
    return out
