"""The work that the row operators beside the selection are judged by: log probabilities of given tokens with entropy and
top alternatives, distillation from a teacher's top logits, and routing to experts, each forward and where it is trained
backward, over the range of shapes and types that they are used with.

`own` chooses whose arithmetic runs: the framework's kernels through its Python entry points, or the same operators in
plain 32-bit torch operations.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


def _logprobs(name, dtype, batch, n, m, k, entropy, temperature=1.0, train=False, mask="none"):
    return {"name": name, "op": "logprobs", "dtype": dtype, "batch": batch, "n": n, "m": m, "k": k, "entropy": entropy,
            "temperature": temperature, "train": train, "mask": mask}


def _distill(name, dtype, batch, n, k, tail, how, temperature=1.0, teacher="bf16", ragged=False):
    return {"name": name, "op": "distill", "dtype": dtype, "batch": batch, "n": n, "k": k, "tail": tail, "how": how,
            "temperature": temperature, "teacher": teacher, "ragged": ragged}


def _route(name, dtype, tokens, experts, k, score, bias, groups, topk_groups, group_score, renormalize, scale, train=False, counts=False):
    return {"name": name, "op": "route", "dtype": dtype, "tokens": tokens, "experts": experts, "k": k, "score": score, "bias": bias,
            "groups": groups, "topk_groups": topk_groups, "group_score": group_score, "renormalize": renormalize, "scale": scale,
            "train": train, "counts": counts}


def listed():
    return [
        # one sequence being decoded: the sampled token's log probability and twenty alternatives; latency is all there is
        _logprobs("logprobs_one_row", "bf16", 1, 131072, 1, 20, False),
        # a small serving batch, with a sampling temperature, entropy for a monitor, and a few alternatives
        _logprobs("logprobs_decode_16", "bf16", 16, 131072, 1, 5, True, 0.7),
        # scoring a prompt: a block of positions, several candidates each; odd rows, none but the first on a 16-byte boundary
        _logprobs("logprobs_prompt_odd", "f32", 300, 50257, 3, 5, False),
        # scoring rollouts for reinforcement learning: the token's log probability and the entropy of every position
        _logprobs("logprobs_score_1024", "bf16", 1024, 131072, 1, 0, True),
        # a policy-gradient step on such rows: forward, then the gradient of both to the logits; odd fp16 rows
        _logprobs("logprobs_train_f16", "f16", 512, 100003, 1, 0, True, train=True),
        # validation of a student on a few positions: the loss alone
        _distill("distill_eval_small", "f16", 8, 30011, 100, False, "forward", teacher="f16"),
        # a training step through automatic differentiation (forward, later backward): teacher lists with the rest as one class
        _distill("distill_tail_odd", "f32", 200, 50257, 50, True, "both", 2.0, "f32", True),
        # the headline of a distillation run: loss and gradient of a block of positions in one call, 1024 teacher logits each
        _distill("distill_step_1024", "bf16", 1024, 131072, 1024, False, "step"),
        # one decoding step of a mixture of experts: sigmoid scores, a balancing bias, groups
        _route("route_decode_16", "bf16", 16, 256, 8, "sigmoid", True, 8, 4, "top2", True, 2.5),
        # the same for a prompt, with the tokens of each expert counted for the dispatch
        _route("route_prompt_16384", "bf16", 16384, 256, 8, "sigmoid", True, 8, 4, "top2", True, 2.5, counts=True),
        # training a small router: softmax scores, no groups, an odd number of experts; forward and backward
        _route("route_train_odd", "f32", 30011, 60, 4, "softmax", False, 1, 1, "max", False, 1.0, train=True),
    ]


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]; mostly not a round one."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.3:
        v = 1 << max(0, v.bit_length() - 1)
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "distill", "distill", "route"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "route":
        tokens = _log(rng, 1, 1 << 16)
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * _log(rng, max(2, 8 // groups), 512 // groups)
        topk_groups = rng.randint(1, groups)
        k = _log(rng, 1, min(16, experts // groups * topk_groups))
        score = rng.choice(["softmax", "sigmoid"])
        c = _route("", dtype, tokens, experts, k, score, score == "sigmoid" and rng.random() < 0.7, groups, topk_groups,
                   "top2" if score == "sigmoid" and groups > 1 and rng.random() < 0.5 else "max", rng.random() < 0.5,
                   rng.choice([1.0, 2.5]), rng.random() < 0.5, rng.random() < 0.5)
    else:
        n = _log(rng, 1 << 10, 1 << 18)
        most = (1 << 27 if dtype != "f32" else 1 << 26) // n
        batch = _log(rng, 1, min(4096, most))
        temperature = rng.choice([1.0, 1.0, 0.7, 2.0])
        if op == "logprobs":
            train = rng.random() < 0.4
            k = 0 if train or rng.random() < 0.3 else _log(rng, 1, 50)
            c = _logprobs("", dtype, batch if not train else max(1, batch // 2), n, _log(rng, 1, 8), k, rng.random() < 0.5, temperature, train,
                          rng.choice(["none", "none", "inf", "lowest"]))
        else:
            how = rng.choice(["forward", "both", "step"])
            c = _distill("", dtype, batch if how == "forward" else max(1, batch // 2), n, _log(rng, 1, min(1024, n // 8)), rng.random() < 0.5, how,
                         temperature, rng.choice(["f32", "bf16", "f16"]), rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _rows(batch, n, g):
    """Logits of a language model's kind: a normal body, eight tokens of a row that stand out."""
    x = torch.empty((batch, n), dtype=torch.float32, device=DEVICE).normal_(0.0, 3.0, generator=g)
    at = torch.randint(0, n, (batch, 8), generator=g, device=DEVICE)
    high = torch.empty((batch, 8), dtype=torch.float32, device=DEVICE).normal_(14.0, 2.0, generator=g)
    return x.scatter_(1, at, high), at


def _prepare_logprobs(case, g):
    batch, n, m = case["batch"], case["n"], case["m"]
    x, at = _rows(batch, n, g)
    # given tokens: mostly ones that stand out, the last a random one
    pick = torch.randint(0, 8, (batch, m), generator=g, device=DEVICE)
    tokens = at.gather(1, pick)
    if m > 1:
        tokens[:, -1] = torch.randint(0, n, (batch,), generator=g, device=DEVICE)
    if case["mask"] != "none":  # a grammar leaves about a third of the vocabulary, the given tokens among it
        low = -math.inf if case["mask"] == "inf" else torch.finfo(TORCH[case["dtype"]]).min
        keep = torch.empty_like(x).uniform_(generator=g) < 0.33
        keep.scatter_(1, tokens, True)
        x = x.masked_fill_(~keep, low)
    s = {"case": case, "logits": x.to(TORCH[case["dtype"]]), "tokens": tokens}
    if case["train"]:  # advantages times a loss scale; a small bonus for entropy
        s["grad_logprobs"] = torch.empty((batch, m), dtype=torch.float32, device=DEVICE).normal_(0.0, 8.0, generator=g)
        s["grad_entropy"] = torch.full((batch,), -0.08, device=DEVICE) if case["entropy"] else None
    return s


def _prepare_distill(case, g):
    batch, n, k = case["batch"], case["n"], case["k"]
    teacher, _ = _rows(batch, n, g)
    student = teacher * 0.8 + torch.empty_like(teacher).normal_(0.0, 1.0, generator=g)
    values, indices = torch.topk(teacher, k, dim=1)
    s = {"case": case, "student": student.to(TORCH[case["dtype"]])}
    del student
    if case["ragged"]:  # lists of different lengths: what is left of a row is padding
        length = k - torch.randint(0, (k + 1) // 2, (batch, 1), generator=g, device=DEVICE)
        indices = torch.where(torch.arange(k, device=DEVICE)[None, :] < length, indices, -1)
    s["values"], s["indices"] = values.to(TORCH[case["teacher"]]), indices
    # (a thousandth more: the values' rounding leaves the teacher's rest above zero)
    s["teacher_lse"] = torch.logsumexp(teacher / case["temperature"], 1) + 1e-3 if case["tail"] else None
    # weights of the positions in the mean over a batch, times a loss scale; one position in eight is padding
    w = torch.empty((batch,), dtype=torch.float32, device=DEVICE).uniform_(0.5, 1.5, generator=g) * 64.0
    s["weights"] = torch.where(torch.arange(batch, device=DEVICE) % 8 == 7, 0.0, w)
    return s


def _prepare_route(case, g):
    tokens, experts = case["tokens"], case["experts"]
    x = torch.empty((tokens, experts), dtype=torch.float32, device=DEVICE).normal_(0.0, 1.5, generator=g)
    x += torch.empty((1, experts), dtype=torch.float32, device=DEVICE).normal_(0.0, 0.5, generator=g)  # some experts are liked
    s = {"case": case, "logits": x.to(TORCH[case["dtype"]]), "bias": None, "counts": None}
    if case["bias"]:
        s["bias"] = torch.empty((experts,), dtype=torch.float32, device=DEVICE).normal_(0.0, 0.1, generator=g)
    if case["train"]:
        s["grad_weights"] = torch.empty((tokens, case["k"]), dtype=torch.float32, device=DEVICE).normal_(generator=g)
    return s


def prepare(case, seed):
    return {"logprobs": _prepare_logprobs, "distill": _prepare_distill, "route": _prepare_route}[case["op"]](case, _generator(seed))


# ---------------------------------------------------------------------------
# the operators in plain operations, in 32 bits
# ---------------------------------------------------------------------------

def _log_softmax(x, temperature):
    y = (x - x.amax(1, keepdim=True)) / temperature
    return y - torch.log(torch.exp(y).sum(1, keepdim=True))


def _plain_logprobs(s):
    case, tokens, k, temperature = s["case"], s["tokens"], s["case"]["k"], s["case"]["temperature"]
    x = s["logits"].float()
    logp = _log_softmax(x, temperature)
    out = {"logprobs": logp.gather(1, tokens)}
    if k:
        indices = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k]
        out["top_logprobs"], out["top_indices"] = logp.gather(1, indices), indices
    if case["entropy"]:
        p = torch.exp(logp)
        plogp = torch.where(p > 0, p * logp, 0.0)
        out["entropy"] = -plogp.sum(1)
    if case["train"]:
        p = torch.exp(logp)
        g = s["grad_logprobs"]
        dx = -p * g.sum(1, keepdim=True)
        if case["entropy"]:
            dx -= s["grad_entropy"][:, None] * (plogp + p * out["entropy"][:, None])
        dx.scatter_add_(1, tokens, g)
        out["grad"] = (dx / temperature).to(s["logits"].dtype)
    return out


def _plain_distill(s):
    case, temperature = s["case"], s["case"]["temperature"]
    x, z = s["student"].float(), s["values"].float()
    given = s["indices"] >= 0
    at = s["indices"].clamp(min=0)
    z = torch.where(given, z, -math.inf)
    logp = _log_softmax(x, temperature)
    logq = z / temperature - s["teacher_lse"][:, None] if case["tail"] else _log_softmax(z, temperature)
    q = torch.exp(logq)
    loss = torch.where(q > 0, q * (logq - logp.gather(1, at)), 0.0).sum(1)
    out = {}
    if case["tail"]:
        rest = (1.0 - q.sum(1)).clamp(min=0.0)
        # the listed places are taken out of the student's sum, not off it
        unlisted = torch.ones_like(x, dtype=torch.bool).scatter_(1, torch.where(given, at, at[:, :1]), False)
        other = torch.where(unlisted, torch.exp(logp), 0.0).sum(1)
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(other)), 0.0)
    out["loss"] = loss
    if case["how"] == "forward":
        return out
    p = torch.exp(logp)
    if case["tail"]:
        dx = p * (q.sum(1) + rest)[:, None] - torch.where(unlisted, p * (rest / other)[:, None], 0.0)
    else:
        dx = p * q.sum(1, keepdim=True)
    dx.scatter_add_(1, at, -q)
    out["grad"] = (dx * (s["weights"] / temperature)[:, None]).to(s["student"].dtype)
    return out


def _plain_route(s):
    case, k, groups = s["case"], s["case"]["k"], s["case"]["groups"]
    x = s["logits"].float()
    if case["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-x))
    else:
        e = torch.exp(x - x.amax(1, keepdim=True))
        score = e / e.sum(1, keepdim=True)
    choice = x
    if case["group_score"] == "top2":
        choice = score
    if case["bias"]:
        choice = score + s["bias"]
    if groups > 1:
        by_group = choice.view(x.shape[0], groups, -1)
        ordered = torch.sort(by_group, dim=2, descending=True)[0]
        of_group = ordered[:, :, 0]
        if case["group_score"] == "top2" and ordered.shape[2] > 1:
            of_group = of_group + ordered[:, :, 1]
        best = torch.sort(of_group, dim=1, descending=True, stable=True)[1][:, : case["topk_groups"]]
        stays = torch.zeros_like(of_group, dtype=torch.bool).scatter_(1, best, True)
        choice = torch.where(stays[:, :, None], by_group, -math.inf).view(x.shape)
    experts = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :k]
    chosen = score.gather(1, experts)
    total = chosen.sum(1, keepdim=True)
    weights = case["scale"] * (chosen / total if case["renormalize"] else chosen)
    out = {"weights": weights, "experts": experts}
    if case["counts"]:
        out["counts"] = torch.zeros(x.shape[1], dtype=torch.int64, device=x.device).scatter_add_(
            0, experts.reshape(-1), torch.ones_like(experts).reshape(-1))
    if case["train"]:
        g = case["scale"] * s["grad_weights"]
        if case["renormalize"]:
            share = chosen / total
            g = (g - (g * share).sum(1, keepdim=True)) / total
        if case["score"] == "sigmoid":
            dx = torch.zeros_like(x).scatter_(1, experts, g * chosen * (1.0 - chosen))
        else:
            dx = (-score * (g * chosen).sum(1, keepdim=True)).scatter_add_(1, experts, g * chosen)
        out["grad"] = dx.to(s["logits"].dtype)
    return out


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _own_logprobs(s):
    from paper_2501_14336_amd import operators as O
    case = s["case"]
    r = O.logprobs(s["logits"], s["tokens"], k=case["k"], temperature=case["temperature"], entropy=case["entropy"])
    out = {"logprobs": r.logprobs}
    if case["k"]:
        out["top_logprobs"], out["top_indices"] = r.top_logprobs, r.top_indices
    if case["entropy"]:
        out["entropy"] = r.entropy
    if case["train"]:
        out["grad"] = O.logprobs_backward(s["logits"], s["tokens"], r.row_stats, s["grad_logprobs"], r.entropy, s["grad_entropy"],
                                          temperature=case["temperature"])
    return out


def _own_distill(s):
    from paper_2501_14336_amd import operators as O
    case = s["case"]
    lists = (s["student"], s["values"], s["indices"])
    how = {"teacher_lse": s["teacher_lse"], "temperature": case["temperature"]}
    if case["how"] == "step":
        loss, grad = O.distill_step(*lists, s["weights"], **how)
        return {"loss": loss, "grad": grad}
    loss, row_stats = O.distill(*lists, **how)
    if case["how"] == "forward":
        return {"loss": loss}
    return {"loss": loss, "grad": O.distill_backward(*lists, row_stats, s["weights"], **how)}


def _own_route(s):
    from paper_2501_14336_amd import operators as O
    case = s["case"]
    counts = torch.zeros(case["experts"], dtype=torch.int64, device=DEVICE) if case["counts"] else None
    weights, experts = O.route(s["logits"], case["k"], score=case["score"], bias=s["bias"], groups=case["groups"],
                               topk_groups=case["topk_groups"], group_score=case["group_score"], renormalize=case["renormalize"],
                               scale=case["scale"], counts=counts)
    out = {"weights": weights, "experts": experts}
    if case["counts"]:
        out["counts"] = counts
    if case["train"]:
        out["grad"] = O.route_backward(s["logits"], experts, s["grad_weights"], score=case["score"], renormalize=case["renormalize"],
                                       scale=case["scale"])
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"logprobs": _own_logprobs, "distill": _own_distill, "route": _own_route}[op](state)
    return {"logprobs": _plain_logprobs, "distill": _plain_distill, "route": _plain_route}[op](state)


def work(case):
    """Logits read once and gradients written once; lists, given tokens and results once each."""
    eb = BYTES[case["dtype"]]
    if case["op"] == "route":
        t, e, k = case["tokens"], case["experts"], case["k"]
        b = t * (e * eb + k * 12) + (4 * e if case["bias"] else 0) + (8 * e if case["counts"] else 0)
        f = t * (e * 4 + k * 8)
        if case["train"]:
            b, f = b + t * (e * eb + k * 4), f + t * e * 3
        return {"bytes": b, "flops": f}
    rows, n, k = case["batch"], case["n"], case["k"]
    if case["op"] == "logprobs":
        b = rows * (n * eb + case["m"] * 12 + k * 12 + (4 if case["entropy"] else 0))
        f = rows * n * (6 if case["entropy"] else 4)
        if case["train"]:  # the gradients of what was returned, and of the logits
            b, f = b + rows * (n * eb + case["m"] * 4 + (4 if case["entropy"] else 0)), f + rows * n * 5
        return {"bytes": b, "flops": f}
    b = rows * (n * eb + k * (8 + BYTES[case["teacher"]]) + 4 + (4 if case["tail"] else 0))
    f = rows * (n * 4 + k * 6)
    if case["how"] != "forward":
        b, f = b + rows * (n * eb + 4), f + rows * n * 4
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_logprobs(case, s):
    y = s["logits"].double() / case["temperature"]
    logp = y - torch.logsumexp(y, dim=1, keepdim=True)
    out = {"logprobs": torch.gather(logp, 1, s["tokens"])}
    if case["k"]:
        out["top_logprobs"] = torch.sort(logp, dim=1, descending=True)[0][:, : case["k"]].contiguous()
        out["top_indices"] = None
    p = logp.exp()
    h = torch.special.entr(p).sum(dim=1)
    if case["entropy"]:
        out["entropy"] = h
    if case["train"]:
        g = s["grad_logprobs"].double()
        grad = torch.zeros_like(y)
        grad.scatter_add_(1, s["tokens"], g)
        grad.sub_(p * g.sum(dim=1, keepdim=True))
        if case["entropy"]:
            grad.add_(s["grad_entropy"].double()[:, None] * (torch.special.entr(p) - p * h[:, None]))
        out["grad"] = grad / case["temperature"]
    return out


def _exact_distill(case, s):
    y = s["student"].double() / case["temperature"]
    batch, n = y.shape
    # the teacher's distribution laid out over the whole row (a place more for the padding)
    place = torch.where(s["indices"] < 0, n, s["indices"])
    z = s["values"].double() / case["temperature"]
    z = z.masked_fill(s["indices"] < 0, -math.inf)
    norm = s["teacher_lse"].double()[:, None] if case["tail"] else torch.logsumexp(z, dim=1, keepdim=True)
    q = torch.zeros((batch, n + 1), dtype=torch.float64, device=y.device).scatter_(1, place, (z - norm).exp())[:, :n]
    logp = torch.log_softmax(y, dim=1)
    loss = (torch.special.xlogy(q, q) - torch.where(q > 0, q * logp, 0.0)).sum(dim=1)
    grad = logp.exp() * q.sum(dim=1, keepdim=True) - q
    if case["tail"]:
        listed = torch.zeros((batch, n + 1), dtype=torch.bool, device=y.device).scatter_(1, place, True)[:, :n]
        left = (1.0 - q.sum(dim=1)).clamp_min(0.0)
        log_other = torch.logsumexp(logp.masked_fill(listed, -math.inf), dim=1)
        loss = loss + torch.special.xlogy(left, left) - torch.where(left > 0, left * log_other, 0.0)
        grad = grad + left[:, None] * (logp.exp() - (logp - log_other[:, None]).exp().masked_fill(listed, 0.0))
    if case["how"] == "forward":
        return {"loss": loss}
    return {"loss": loss, "grad": grad * s["weights"].double()[:, None] / case["temperature"]}


def _exact_route(case, s):
    x = s["logits"].double()
    rows, e = x.shape
    score = torch.sigmoid(x) if case["score"] == "sigmoid" else torch.softmax(x, dim=1)
    rank = score + s["bias"].double() if case["bias"] else score if case["group_score"] == "top2" else x
    if case["groups"] > 1:
        size = e // case["groups"]
        parts = rank.reshape(rows, case["groups"], size)
        value = torch.topk(parts, min(2 if case["group_score"] == "top2" else 1, size), dim=2)[0].sum(dim=2)
        order = torch.argsort(value, dim=1, descending=True, stable=True)
        out_of = torch.ones_like(value, dtype=torch.bool).scatter_(1, order[:, : case["topk_groups"]], False)
        rank = rank.masked_fill(out_of.repeat_interleave(size, dim=1), -math.inf)
    at = torch.argsort(rank, dim=1, descending=True, stable=True)[:, : case["k"]]
    logits = x.clone().requires_grad_(case["train"])
    again = torch.sigmoid(logits) if case["score"] == "sigmoid" else torch.softmax(logits, dim=1)
    w = torch.gather(again, 1, at)
    if case["renormalize"]:
        w = w / w.sum(dim=1, keepdim=True)
    w = w * case["scale"]
    out = {"weights": w.detach(), "experts": None}
    if case["counts"]:
        out["counts"] = None
    if case["train"]:
        out["grad"] = torch.autograd.grad((w * s["grad_weights"].double()).sum(), logits)[0]
    return out


def exact(case, seed):
    """What run() returns, in 64 bits; whole numbers have no such value."""
    s = prepare(case, seed)
    return {"logprobs": _exact_logprobs, "distill": _exact_distill, "route": _exact_route}[case["op"]](case, s)
