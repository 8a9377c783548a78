"""The work that the operators on logits are judged on: log probabilities of given tokens (with entropy and the top
alternatives) and their gradient, and distillation from a teacher's top logits, forward and backward.

`listed()` names the fixed cases, `draw(rng)` gives further ones of the same ranges, `prepare` makes what a program has in
hand before the call, `run` is one pass: the framework's entry points where `own` is true, else the same formulas in
elementary torch operations in 32 bits.  `exact` is the definition in 64 bits, `work` the bytes and operations that a
pass cannot do without.

Operators (the "op" of a case):
  logprobs        scores of given tokens, and what the case asks for besides: entropy, the k best alternatives
  logprobs_train  the same scores (and entropy) as a differentiable loss term: values and the gradient of the logits
  distill         loss against a teacher's list and the gradient of the logits in one call, rows weighted
  distill_train   the same loss as a differentiable term: values and the gradient of the logits
"""
import math

import torch

own = False

PAD = -100  # a position without a token to score: a prompt's, or padding


def listed():
    return [
        # one new token: its log probability and twenty alternatives, as a serving interface returns them
        {"name": "logprobs_t1", "op": "logprobs", "T": 1, "V": 50257, "stride": 50257, "dtype": "bf16", "k": 20,
         "temperature": 1.0, "entropy": True, "masked": False, "pad": 0.0},
        # one decoding step of 64 sequences with fp32 logits, five alternatives, sampled below temperature 1
        {"name": "logprobs_t64_f32", "op": "logprobs", "T": 64, "V": 50257, "stride": 50257, "dtype": "f32", "k": 5,
         "temperature": 0.7, "entropy": False, "masked": False, "pad": 0.0},
        # constrained decoding in a padded vocabulary: masks of -inf and of the type's lowest value, rows left empty
        {"name": "logprobs_masked_t333", "op": "logprobs", "T": 333, "V": 32003, "stride": 32064, "dtype": "bf16", "k": 10,
         "temperature": 1.0, "entropy": True, "masked": True, "pad": 0.1},
        # a large vocabulary of odd size, a long list
        {"name": "logprobs_wide_t96", "op": "logprobs", "T": 96, "V": 200003, "stride": 200003, "dtype": "bf16", "k": 100,
         "temperature": 1.3, "entropy": True, "masked": False, "pad": 0.0},
        # a teacher's pass over 2048 tokens in fp32: the 64 best logits of every position and the log sum
        {"name": "teacher_t2048_f32", "op": "logprobs", "T": 2048, "V": 50257, "stride": 50257, "dtype": "f32", "k": 64,
         "temperature": 2.0, "entropy": False, "masked": False, "pad": 0.0},
        # scoring of 8 sequences of 512 tokens (perplexity): nothing but the tokens' log probabilities
        {"name": "score_t4096", "op": "logprobs", "T": 4096, "V": 50257, "stride": 50257, "dtype": "bf16", "k": 0,
         "temperature": 1.0, "entropy": False, "masked": False, "pad": 0.0},
        # the usual training loss on the same batch, a quarter of the positions being prompts
        {"name": "nll_train_t4096", "op": "logprobs_train", "T": 4096, "V": 50257, "stride": 50257, "dtype": "bf16",
         "temperature": 1.0, "entropy": False, "masked": False, "pad": 0.25},
        # log probabilities with an entropy bonus, fp32 logits of an odd vocabulary
        {"name": "entropy_train_t777_f32", "op": "logprobs_train", "T": 777, "V": 30011, "stride": 30011, "dtype": "f32",
         "temperature": 0.8, "entropy": True, "masked": False, "pad": 0.1},
        # a short answer distilled: 24 tokens, the teacher's list alone
        {"name": "distill_t24", "op": "distill", "T": 24, "V": 50257, "stride": 50257, "dtype": "bf16", "k": 20,
         "temperature": 1.0, "rest": False, "pad": 0.0},
        # fp32 logits, a list of 32 renormalised
        {"name": "distill_t2048_f32", "op": "distill", "T": 2048, "V": 50257, "stride": 50257, "dtype": "f32", "k": 32,
         "temperature": 1.0, "rest": False, "pad": 0.1},
        # as a term of an automatically differentiated loss, with the rest of the teacher's vocabulary as one outcome
        {"name": "distill_train_t1000", "op": "distill_train", "T": 1000, "V": 50257, "stride": 50304, "dtype": "bf16", "k": 16,
         "temperature": 2.0, "rest": True, "pad": 0.0},
        # the largest: 8 sequences of 2048 tokens, 64 logits of the teacher and the rest
        {"name": "distill_t16384", "op": "distill", "T": 16384, "V": 50257, "stride": 50257, "dtype": "bf16", "k": 64,
         "temperature": 2.0, "rest": True, "pad": 0.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "logprobs", "logprobs_train", "logprobs_train", "distill", "distill",
                     "distill_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    size = 2 if dtype == "bf16" else 4
    V = _log(rng, 4000, 250000)
    T = _log(rng, 1, 16384)
    while T * V * size > 16384 * 50257 * 2:  # no more than the largest listed case
        T = _log(rng, 1, 16384)
    stride = V if rng.random() < 0.6 else -(-V // 64) * 64 + rng.choice([0, 0, 64, 3])
    case = {"op": op, "T": T, "V": V, "stride": stride, "dtype": dtype, "pad": rng.choice([0.0, 0.0, 0.1, 0.5]),
            "temperature": rng.choice([1.0, 1.0, 0.5, 0.8, 1.5, 2.0, 4.0])}
    if op == "logprobs":
        case.update(k=rng.choice([0, 1, _log(rng, 2, 20), _log(rng, 20, 128)]), entropy=rng.random() < 0.5,
                    masked=rng.random() < 0.25)
    elif op == "logprobs_train":
        case.update(entropy=rng.random() < 0.4, masked=rng.random() < 0.25)
    else:
        case.update(k=_log(rng, 4, 128), rest=rng.random() < 0.5)
    if case.get("masked"):  # the lowest value of a type stays within the type
        case["temperature"] = max(1.0, case["temperature"])
    return case


# ---- inputs -----------------------------------------------------------------------------------------------------

def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _logits(case, gen):
    """Rows of a trained model's kind: a broad body (spread 2.5) and a few words far above it, in rows of `stride`."""
    T, V = case["T"], case["V"]
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    buf = torch.randn((T, case["stride"]), generator=gen, device="cuda").mul_(2.5)
    peaks = torch.randint(V, (T, 8), generator=gen, device="cuda")
    buf.scatter_(1, peaks, 10.0 * torch.rand((T, 8), generator=gen, device="cuda") + 4.0)
    x = buf.to(dtype)[:, :V]
    if case.get("masked"):
        # half the rows keep a twentieth of the vocabulary, every eighth keeps 7 entries, every eighth none; the masks'
        # value is -inf, or the type's lowest in half of the rows that keep much or nothing
        r = torch.arange(T, device="cuda")[:, None]
        fill = torch.where((r % 2 == 0) | (r % 8 == 5), float("-inf"), torch.finfo(dtype).min).to(dtype)
        drop = (torch.rand((T, V), generator=gen, device="cuda") > 0.05) & (r % 4 >= 2)
        few = torch.ones((T, V), dtype=torch.bool, device="cuda")
        few.scatter_(1, torch.randint(V, (T, 7), generator=gen, device="cuda"), False)
        drop = torch.where(r % 16 >= 14, True, torch.where(r % 8 == 5, few, drop))
        x.copy_(torch.where(drop, fill, x))
    return x


def _tokens(case, x, gen):
    """One token a row, half of them (all where a mask allows few) the likeliest, `pad` of the rows without one."""
    T, V = x.shape
    likely = torch.rand((T,), generator=gen, device="cuda") < (1.0 if case["masked"] else 0.5)
    token = torch.where(likely, x.argmax(1), torch.randint(V, (T,), generator=gen, device="cuda"))
    return torch.where(torch.rand((T,), generator=gen, device="cuda") < case["pad"], PAD, token)


def prepare(case, seed):
    gen = _generator(seed)
    T = case["T"]
    x = _logits(case, gen)
    state = {"case": case, "x": x}
    if case["op"].startswith("logprobs"):
        state["tokens"] = _tokens(case, x, gen)
    else:
        # the teacher agrees with the student in part; its list and log sum at the loss's temperature are kept
        k, c = case["k"], 1.0 / case["temperature"]
        z = torch.randn(x.shape, generator=gen, device="cuda").mul_(1.5).add_(x, alpha=0.8)
        best = z.topk(k, dim=1)
        state.update(top_logit=best.values, top_index=best.indices.to(torch.int32),
                     teacher_lse=torch.logsumexp(z.mul_(c), dim=1) if case["rest"] else None)
    keep = torch.rand((T,), generator=gen, device="cuda") >= case["pad"]
    if case["op"] == "distill":
        state["weight"] = keep.float() / T
    elif case["op"] == "distill_train":
        state["dloss"] = torch.rand((T,), generator=gen, device="cuda").add_(0.5).mul_(keep) / T
    elif case["op"] == "logprobs_train":
        state["dlogp"] = -torch.rand((T,), generator=gen, device="cuda").add_(0.5) / T
        if case["entropy"]:
            state["dentropy"] = torch.full((T,), -0.01 / T, device="cuda")
    if case["op"].endswith("_train"):
        x.requires_grad_(True)
    return state


# ---- the formulas in elementary operations, in the type of `x` (32 bits in the plain form) ---------------------------

def _softmax_parts(x, c):
    """d = (x - max) c, e = exp(d), S = sum e; a row of -inf alone has S = 0."""
    m = x.max(1, keepdim=True).values
    m = torch.where(m == float("-inf"), 0.0, m)
    d = (x - m) * c
    e = torch.exp(d)
    return m[:, 0], d, e, e.sum(1)


def _scores(x, tokens, c, want_entropy):
    m, d, e, S = _softmax_parts(x, c)
    logS = torch.log(S)
    empty = S == 0
    given = tokens >= 0
    at = torch.where(given, tokens, 0)[:, None]
    logp = d.gather(1, at)[:, 0] - logS
    logp = torch.where(given, torch.where(empty, float("-inf"), logp), 0.0)
    entropy = None
    if want_entropy:
        weighted = torch.where(e == 0, 0.0, e * d).sum(1)
        entropy = torch.where(empty, 0.0, logS - weighted / S)
    return m, d, e, S, logS, empty, given, at, logp, entropy


def _plain_top(x, k):
    """The k best of every row, the lowest index first among equals."""
    bits = (x + 0.0).view(torch.int32)  # -0 counts as 0
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
    key = order * (1 << 21) + ((1 << 21) - 1 - torch.arange(x.shape[1], device=x.device))
    best = key.topk(k, dim=1).values
    return (1 << 21) - 1 - (best & ((1 << 21) - 1))


def _plain_logprobs(case, state):
    c = 1.0 / case["temperature"]
    x = state["x"].float()
    m, d, e, S, logS, empty, _, _, logp, entropy = _scores(x, state["tokens"], c, case["entropy"])
    out = {"logp": logp, "lse": torch.where(empty, float("-inf"), m * c + logS)}
    if entropy is not None:
        out["entropy"] = entropy
    if case["k"]:
        index = _plain_top(x, case["k"])
        out["top_index"] = index.to(torch.int32)
        out["top_logit"] = x.gather(1, index)
        out["top_logp"] = torch.where(empty[:, None], float("-inf"), d.gather(1, index) - logS[:, None])
    return out


def _logprobs_gradient(x, tokens, c, dlogp, dentropy):
    m, d, e, S, logS, empty, given, at, logp, entropy = _scores(x, tokens, c, dentropy is not None)
    q = e / torch.where(empty, 1.0, S)[:, None]
    g = torch.where(given & ~empty, dlogp, 0.0)
    dx = -q * g[:, None]
    dx.scatter_add_(1, at, g[:, None])
    if dentropy is not None:
        logq = torch.where(e == 0, 0.0, d - logS[:, None])
        dx -= dentropy[:, None] * q * torch.where(e == 0, 0.0, logq + entropy[:, None])
    return logp, entropy, dx * c


def _distill(x, top_logit, top_index, teacher_lse, c, weight):
    """Loss of every row and the gradient of sum(weight * loss)."""
    index = top_index.to(torch.int64)
    z = top_logit * c
    if teacher_lse is None:
        top = z.max(1, keepdim=True).values
        teacher_lse = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))[:, 0]
        rest = None
    else:
        rest = torch.clamp(1.0 - torch.exp(z - teacher_lse[:, None]).sum(1), min=0.0)
    logp = z - teacher_lse[:, None]
    p = torch.exp(logp)
    m, d, e, S = _softmax_parts(x, c)
    logq = d.gather(1, index) - torch.log(S)[:, None]
    loss = (p * (logp - logq)).sum(1)
    q = e / S[:, None]
    if rest is None:
        dx = q * p.sum(1, keepdim=True)
        listed_dx = torch.exp(logq) * p.sum(1, keepdim=True) - p
    else:
        e.scatter_(1, index, 0.0)
        qbar = e.sum(1) / S
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - torch.log(qbar)), 0.0)
        dx = q * (1.0 - rest / qbar)[:, None]
        listed_dx = torch.exp(logq) - p
    dx.scatter_(1, index, listed_dx)
    dx *= (weight / c)[:, None]
    return loss / (c * c), dx


def _plain(state):
    case = state["case"]
    c, dtype = 1.0 / case["temperature"], state["x"].dtype
    if case["op"] == "logprobs":
        return _plain_logprobs(case, state)
    x = state["x"].detach().float()
    if case["op"] == "logprobs_train":
        logp, entropy, dx = _logprobs_gradient(x, state["tokens"], c, state["dlogp"], state.get("dentropy"))
        return [logp] + ([entropy] if entropy is not None else []) + [dx.to(dtype)]
    weight = state["weight"] if case["op"] == "distill" else state["dloss"]
    loss, dx = _distill(x, state["top_logit"], state["top_index"], state["teacher_lse"], c, weight)
    if case["op"] == "distill":  # rows of weight 0 are skipped
        loss = torch.where(weight == 0, 0.0, loss)
    return [loss, dx.to(dtype)]


def _own(state):
    import paper_2210_03858_amd as bcq
    from paper_2210_03858_amd import autograd
    case, x = state["case"], state["x"]
    temperature = case["temperature"]
    if case["op"] == "logprobs":
        out = bcq.bcq_logprobs_fwd(x, state["tokens"], k=case["k"], temperature=temperature, entropy=case["entropy"], lse=True)
        return {name: t for name, t in out._asdict().items() if t is not None}
    if case["op"] == "logprobs_train":
        logp, entropy = autograd.token_logprobs(x, state["tokens"], temperature=temperature, entropy=case["entropy"])
        if entropy is None:
            return [logp.detach(), torch.autograd.grad(logp, x, state["dlogp"])[0]]
        dx = torch.autograd.grad((logp, entropy), x, (state["dlogp"], state["dentropy"]))[0]
        return [logp.detach(), entropy.detach(), dx]
    if case["op"] == "distill":
        return list(bcq.bcq_distill_fwd_bwd(x, state["top_logit"], state["top_index"], weight=state["weight"],
                                            teacher_lse=state["teacher_lse"], temperature=temperature))
    loss = autograd.distill_loss(x, state["top_logit"], state["top_index"], teacher_lse=state["teacher_lse"],
                                 temperature=temperature)
    return [loss.detach(), torch.autograd.grad(loss, x, state["dloss"])[0]]


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits, written apart from the plain form ------------------------------------------------------

def _rows(T, V, elements=1 << 26):
    """Row blocks of a bounded number of elements."""
    step = max(1, elements // V)
    return [slice(t, min(T, t + step)) for t in range(0, T, step)]


def exact(case, seed):
    state = prepare(case, seed)
    x, tau = state["x"].detach(), float(case["temperature"])
    T, V = x.shape
    parts = []
    for rows in _rows(T, V):
        y = x[rows].double() / tau
        n = y.shape[0]
        top = y.amax(1)
        y -= torch.where(torch.isfinite(top), top, 0.0)[:, None]  # 64 bits hold no sum of the lowest value and a logarithm
        L = torch.logsumexp(y, 1)
        alive = torch.isfinite(L)
        logq = torch.where(alive[:, None], y - L[:, None], float("-inf"))
        if case["op"].startswith("logprobs"):
            tok = state["tokens"][rows]
            here = torch.where(tok < 0, 0.0, logq[torch.arange(n, device="cuda"), tok.clamp(min=0)])
            H = torch.special.entr(logq.exp()).sum(1) if case["entropy"] else None
            if case["op"] == "logprobs":
                part = {"logp": here, "lse": torch.where(alive, L + top, top)}
                if H is not None:
                    part["entropy"] = H
                if case["k"]:
                    part["top_logit"] = x[rows].double().topk(case["k"], 1).values
                    part["top_logp"] = logq.topk(case["k"], 1).values
                parts.append(part)
                continue
            q = logq.exp()
            g = (state["dlogp"][rows].double() * (tok >= 0) * alive)[:, None]
            unit = torch.zeros_like(q).scatter_(1, tok.clamp(min=0)[:, None], 1.0)
            grad = g * (unit - q)
            if H is not None:
                grad += state["dentropy"][rows].double()[:, None] * (torch.special.entr(q) - q * H[:, None])
            parts.append([here] + ([H] if H is not None else []) + [grad / tau])
            continue
        j = state["top_index"][rows].long()
        lp = state["top_logit"][rows].double() / tau
        lp = lp - (torch.logsumexp(lp, 1) if state["teacher_lse"] is None else state["teacher_lse"][rows].double())[:, None]
        p = lp.exp()
        inside = torch.zeros((n, V), dtype=torch.bool, device="cuda").scatter_(1, j, True)
        target = torch.zeros_like(logq).scatter_(1, j, p)
        loss = (p * (lp - logq.gather(1, j))).sum(1)
        if state["teacher_lse"] is not None:
            r = (1.0 - p.sum(1)).clamp(min=0.0)
            lrest = torch.logsumexp(logq.masked_fill(inside, float("-inf")), 1)
            loss += torch.where(r > 0, r * (r.log() - lrest), 0.0)
            target += torch.where(inside, 0.0, r[:, None] * (logq - lrest[:, None]).exp())
        w = (state["weight"] if case["op"] == "distill" else state["dloss"])[rows].double()
        if case["op"] == "distill":
            loss = torch.where(w == 0, 0.0, loss)
        parts.append([loss * tau * tau, (logq.exp() - target) * (w * tau)[:, None]])
    if case["op"] == "logprobs":
        names = ["logp", "lse"] + ["entropy"] * bool(case["entropy"]) + ["top_index", "top_logit", "top_logp"] * bool(case["k"])
        return {name: None if name == "top_index" else torch.cat([p[name] for p in parts]) for name in names}
    return [torch.cat(column) for column in zip(*parts)]


def work(case):
    T, V = case["T"], case["V"]
    size = 2.0 if case["dtype"] == "bf16" else 4.0
    table = T * V * size
    k = case.get("k", 0)
    if case["op"] == "logprobs":
        # a maximum, a difference, a product, an exponential and a sum an entry; entropy: a product and a sum; a comparison
        return {"bytes": table + T * (8 + 8 + 4 * bool(case["entropy"]) + 12 * k),
                "flops": T * V * (5.0 + 2.0 * bool(case["entropy"]) + 1.0 * bool(k))}
    # logits in, gradient out; rows that are skipped are not read
    alive = 1.0 - (case["pad"] if not case.get("entropy") else 0.0)
    return {"bytes": table * (1.0 + alive) + T * (16 + 8 * k), "flops": T * V * alive * (8.0 + 4.0 * bool(case.get("entropy")))}
