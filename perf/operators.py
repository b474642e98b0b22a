"""Cases for the operators over a vocabulary: log probabilities of given tokens (with entropy and top alternatives),
their backward pass, and distillation from a teacher's top logits with its gradient.

``run`` computes a case either in plain torch operations (32 bits, one rounding at the end) or, where ``own`` is
true, through the library's entry points; ``exact`` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False
_module = None


def _qn():
    global _module
    if _module is None:
        from paper_1709_05069_b200 import qn

        _module = qn
    return _module


_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def _case(name, op, rows, vocab, dtype, k=0, temperature=1.0, pad=0, **more):
    case = {"name": name, "op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "k": k, "temperature": temperature,
            "pad": pad, "constrained": False, "skip": 0, "entropy": True, "teacher": "logprobs", "grad": True}
    case.update(more)
    return case


def listed():
    return [
        # one token of one sequence, as an answer is sampled: latency is all that counts; a quarter of the vocabulary
        # range of common tokenizers
        _case("logprobs_one_token", "logprobs", 1, 32768, "bf16", 8, 0.7),
        # one decoding step of a batch, with the 20 alternatives that serving interfaces report; some rows are
        # constrained to a grammar (nine tenths of the vocabulary at -inf)
        _case("logprobs_decode_batch", "logprobs", 96, 131072, "bf16", 20, 0.7, constrained=True),
        # scoring a prompt's tokens in evaluation: fp32 logits, an odd vocabulary (no row but the first is aligned)
        _case("logprobs_prompt_odd", "logprobs", 1023, 50001, "f32", 1),
        # a teacher's top 64 written down for a batch of training sequences: the largest forward pass
        _case("logprobs_teacher_dump", "logprobs", 8192, 131072, "bf16", 64),
        # gradient of a short answer's tokens with alternatives and an entropy term: fp32, odd sizes
        _case("backward_small_odd", "backward", 77, 20011, "f32", 5, 0.7),
        # policy-gradient step: upstream gradients of log probability and entropy
        _case("backward_policy", "backward", 4096, 131072, "bf16", 0),
        # negative log-likelihood of ragged sequences packed into a batch: an eighth of the rows are padding (their
        # upstream gradient is 0), odd vocabulary, no entropy term
        _case("backward_ragged_odd", "backward", 2047, 100003, "bf16", 0, skip=8, entropy=False),
        # one small Worker's minibatch
        _case("distill_small", "distill", 4, 8192, "f32", 16, teacher="logits"),
        # a training step: loss and gradient against a stored teacher's top 64 log probabilities
        _case("distill_step", "distill", 4096, 131072, "bf16", 64),
        # softened distillation over ragged sequences, logits stored with padded rows of an odd vocabulary
        _case("distill_ragged_odd", "distill", 1500, 65537, "bf16", 32, 2.0, pad=7, skip=8, teacher="logits"),
        # the largest vocabulary in fp32, with a long list
        _case("distill_f32_large", "distill", 1024, 262144, "f32", 128),
        # the loss alone, on held-out data
        _case("distill_eval", "distill", 2048, 32000, "bf16", 20, grad=False),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "backward", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    vocab = _log_uniform(rng, 512, 262144)
    if rng.random() < 0.5:
        vocab = max(512, vocab // 128 * 128)
    most = ((1 << 30) if op == "logprobs" else (1 << 29)) * 2 // _BYTES[dtype] // vocab
    rows = min(_log_uniform(rng, 1, 8192), most)
    case = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "k": _log_uniform(rng, 1, 128),
            "temperature": rng.choice([1.0, 1.0, 0.7, 2.0]), "pad": rng.choice([0, 0, 8, 64, rng.randrange(1, 64)]),
            "constrained": False, "skip": 0, "entropy": rng.random() < 0.5, "teacher": "logprobs", "grad": True}
    if op == "logprobs":
        case["k"] = rng.choice([0, case["k"], case["k"]])
        case["constrained"] = rng.random() < 0.3
    else:
        case["skip"] = rng.choice([0, 0, 4, 8])
        if op == "backward":
            case["k"] = rng.choice([0, 0, case["k"]])
        else:
            case["teacher"] = rng.choice(["logits", "logprobs"])
            case["grad"] = rng.random() < 0.8
    return case


def _kept_rows(case):
    """Rows that count: with ``skip`` = s every s-th row is padding."""
    return case["rows"] - (case["rows"] // case["skip"] if case["skip"] else 0)


def work(case):
    rows, vocab, k, size = case["rows"], case["vocab"], case["k"], _BYTES[case["dtype"]]
    kept = _kept_rows(case)
    if case["op"] == "logprobs":  # tokens in; logprob, lse, entropy, alternatives out; sub, scale, exp, add, fma
        return {"bytes": rows * vocab * size + rows * (8 + 12 + 12 * k), "flops": 6 * rows * vocab}
    if case["op"] == "backward":
        return {"bytes": (kept + rows) * vocab * size + rows * (8 + 4 + (4 if case["entropy"] else 0) + 12 * k),
                "flops": (11 if case["entropy"] else 8) * kept * vocab}
    out = rows * vocab * size if case["grad"] else 0
    return {"bytes": kept * vocab * size + out + rows * (8 + 12 * k), "flops": (9 if case["grad"] else 5) * kept * vocab}


def _logits(case, gen):
    """Logits as a language model gives them: a spread of a few units around a falling unigram prior."""
    rows, vocab, dtype = case["rows"], case["vocab"], _DTYPES[case["dtype"]]
    order = torch.randperm(vocab, generator=gen, device="cuda")
    prior = -0.8 * torch.log1p(order.float())
    store = torch.empty((rows, vocab + case["pad"]), dtype=dtype, device="cuda")
    store.normal_(0.0, 2.5, generator=gen)
    store[:, :vocab] += prior.to(dtype)
    logits = store[:, :vocab]
    if case["constrained"]:  # every fourth row may only use a tenth of the vocabulary
        allowed = torch.rand((logits[::4].shape[0], vocab), generator=gen, device="cuda") < 0.1
        allowed[:, :2] = True
        logits[::4] = torch.where(allowed, logits[::4], torch.full((), -math.inf, dtype=dtype, device="cuda"))
    return logits


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    rows, vocab, k, dtype = case["rows"], case["vocab"], case["k"], _DTYPES[case["dtype"]]
    s = {"case": case, "logits": _logits(case, gen)}

    def vector(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda")

    def upstream(*shape):
        return torch.randn(shape, generator=gen, device="cuda") / rows

    padding = torch.zeros(rows, dtype=torch.bool, device="cuda")
    if case["skip"]:
        padding[case["skip"] - 1::case["skip"]] = True
    if case["op"] in ("logprobs", "backward"):
        # given tokens: drawn from the model's own distribution (argmax of logits / T + Gumbel noise), as an answer's
        # tokens are, by blocks of rows
        tokens = torch.empty(rows, dtype=torch.int64, device="cuda")
        for a in range(0, rows, 512):
            z = s["logits"][a:a + 512].float() / case["temperature"]
            tokens[a:a + 512] = (z - torch.empty_like(z).exponential_(1.0, generator=gen).log()).argmax(1)
        s["tokens"] = tokens
    if case["op"] == "logprobs":
        s["logprob"], s["lse"], s["entropy"] = vector(rows), vector(rows), vector(rows)
        if k:
            s["top_token"] = torch.empty((rows, k), dtype=torch.int64, device="cuda")
            s["top_logprob"] = vector(rows, k)
    elif case["op"] == "backward":
        # upstream gradients, and the alternatives that the forward pass named
        if k:
            s["top_token"] = torch.empty((rows, k), dtype=torch.int64, device="cuda")
            for a in range(0, rows, 512):
                s["top_token"][a:a + 512] = s["logits"][a:a + 512].topk(k, 1).indices
        s["d_logprob"] = upstream(rows).masked_fill(padding, 0.0)
        s["d_entropy"] = upstream(rows).masked_fill(padding, 0.0) if case["entropy"] else None
        s["d_top_logprob"] = upstream(rows, k).masked_fill(padding[:, None], 0.0) if k else None
        s["dlogits"] = torch.empty((rows, vocab), dtype=dtype, device="cuda")
    else:
        # the teacher sees the same text: its logits are the student's with some disagreement
        s["teacher_token"] = torch.empty((rows, k), dtype=torch.int64, device="cuda")
        s["teacher_value"] = vector(rows, k)
        for a in range(0, rows, 512):
            z = s["logits"][a:a + 512].float()
            z = (z + 0.7 * torch.randn(z.shape, generator=gen, device="cuda")) / case["temperature"]
            top = z.topk(k, 1)
            s["teacher_token"][a:a + 512] = top.indices
            s["teacher_value"][a:a + 512] = (top.values - torch.logsumexp(z, 1, keepdim=True)
                                             if case["teacher"] == "logprobs" else top.values * case["temperature"])
        s["weight"] = torch.full((rows,), 1.0 / _kept_rows(case), device="cuda").masked_fill(padding, 0.0)
        s["loss"] = vector(rows)
        s["dlogits"] = torch.empty((rows, vocab), dtype=dtype, device="cuda") if case["grad"] else None
    return s


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _plain_logprobs(s):
    case, z = s["case"], s["logits"].float()
    u = z / case["temperature"]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    total = e.sum(1, keepdim=True)
    shift = torch.log(total)
    out = {"logprob": (u.gather(1, s["tokens"][:, None]) - shift)[:, 0],
           "lse": (z.amax(1, keepdim=True) / case["temperature"] + shift)[:, 0],
           "entropy": (shift - torch.where(e > 0, e * u, 0.0).sum(1, keepdim=True) / total)[:, 0]}
    if case["k"]:
        # one key for each logit, larger for a larger logit and, among equals, for a lower index
        bits = (z + 0.0).view(torch.int32)
        order = bits ^ ((bits >> 31) & 0x7FFFFFFF)
        last = z.shape[1] - 1
        key = (order.to(torch.int64) << 32) + (last - torch.arange(last + 1, device="cuda"))
        kept = min(case["k"], last + 1)
        top = last - (key.topk(kept, 1).values & 0xFFFFFFFF)
        value = u.gather(1, top) - shift
        out["top_token"] = torch.where(value > -math.inf, top, -1)
        out["top_logprob"] = value
    return out


def _plain_backward(s):
    case = s["case"]
    u = s["logits"].float() / case["temperature"]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    total = e.sum(1, keepdim=True)
    p = e / total
    a = -s["d_logprob"]
    if case["k"]:
        a = a - s["d_top_logprob"].sum(1)
    if s["d_entropy"] is not None:
        logp = u - torch.log(total)
        entropy = -(p * logp).sum(1, keepdim=True)
        d = p * (a[:, None] - s["d_entropy"][:, None] * (logp + entropy))
    else:
        d = p * a[:, None]
    d.scatter_add_(1, s["tokens"][:, None], s["d_logprob"][:, None])
    if case["k"]:
        d.scatter_add_(1, s["top_token"], s["d_top_logprob"])
    return {"dlogits": (d / case["temperature"]).to(s["logits"].dtype)}


def _plain_distill(s):
    case, w = s["case"], s["weight"][:, None]
    token, value = s["teacher_token"], s["teacher_value"]
    u = s["logits"].float() / case["temperature"]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    total = e.sum(1, keepdim=True)
    logp = u.gather(1, token) - torch.log(total)
    if case["teacher"] == "logits":
        v = value / case["temperature"]
        v = v - v.amax(1, keepdim=True)
        logq = v - torch.log(torch.exp(v).sum(1, keepdim=True))
        q = torch.exp(logq)
        loss = (q * (logq - logp)).sum(1)
        d = e * (q.sum(1, keepdim=True) / total) if case["grad"] else None
    else:
        q = torch.exp(value)
        q_rest = torch.clamp(1.0 - q.sum(1, keepdim=True), min=0.0)
        rest = e.scatter(1, token, 0.0)
        rest_total = rest.sum(1, keepdim=True)
        tail = torch.where(q_rest > 0, q_rest * (torch.log(q_rest) - torch.log(rest_total / total)), 0.0)
        loss = (q * (value - logp)).sum(1) + tail[:, 0]
        d = e * ((q.sum(1, keepdim=True) + q_rest) / total) - rest * (q_rest / rest_total) if case["grad"] else None
    out = {"loss": torch.where(w[:, 0] != 0, loss, 0.0)}
    if case["grad"]:
        d.scatter_add_(1, token, -q)
        out["dlogits"] = (d * (w / case["temperature"])).to(s["logits"].dtype)
    return out


# ---- the library's calls -------------------------------------------------------------------------------------------


def _own_logprobs(s):
    case = s["case"]
    top_token, top_logprob = s.get("top_token"), s.get("top_logprob")
    _qn().qn_logprobs(s["logits"], s["tokens"], s["logprob"], lse=s["lse"], entropy=s["entropy"], top_token=top_token,
                      top_logprob=top_logprob, temperature=case["temperature"])
    out = {"logprob": s["logprob"], "lse": s["lse"], "entropy": s["entropy"]}
    if top_token is not None:
        out["top_token"], out["top_logprob"] = top_token, top_logprob
    return out


def _own_backward(s):
    _qn().qn_logprobs_backward(s["logits"], s["dlogits"], tokens=s["tokens"], d_logprob=s["d_logprob"],
                               d_entropy=s["d_entropy"], top_token=s.get("top_token"),
                               d_top_logprob=s["d_top_logprob"], temperature=s["case"]["temperature"])
    return {"dlogits": s["dlogits"]}


def _own_distill(s):
    qn, case = _qn(), s["case"]
    qn.qn_distill(s["logits"], s["teacher_token"], s["teacher_value"], s["loss"], dlogits=s["dlogits"],
                  weight=s["weight"], temperature=case["temperature"],
                  teacher=qn.QN_TEACHER_LOGITS if case["teacher"] == "logits" else qn.QN_TEACHER_LOGPROBS)
    return {"loss": s["loss"], "dlogits": s["dlogits"]} if case["grad"] else {"loss": s["loss"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_logprobs if op == "logprobs" else _own_backward if op == "backward" else _own_distill)(state)
    return (_plain_logprobs if op == "logprobs" else _plain_backward if op == "backward" else _plain_distill)(state)


# ---- 64 bits -------------------------------------------------------------------------------------------------------


def _exact_rows(s, a, b):
    """The outputs for rows a..b from the definitions, in float64: probabilities first, everything from them."""
    case, t = s["case"], s["case"]["temperature"]
    z = s["logits"][a:b].double()
    logp = torch.log_softmax(z / t, 1)
    p = logp.exp()
    each = torch.arange(b - a, device="cuda")
    if case["op"] == "logprobs":
        out = {"logprob": logp[each, s["tokens"][a:b]], "lse": torch.logsumexp(z / t, 1),
               "entropy": torch.special.entr(p).sum(1)}
        if case["k"]:
            out["top_logprob"] = logp.topk(min(case["k"], z.shape[1]), 1).values
        return out
    if case["op"] == "backward":
        # chain rule through log_softmax: d(logp) -> d(u) = d(logp) - p * sum d(logp)
        d = torch.zeros_like(p)
        d[each, s["tokens"][a:b]] += s["d_logprob"][a:b].double()
        if case["k"]:
            d.scatter_add_(1, s["top_token"][a:b], s["d_top_logprob"][a:b].double())
        if s["d_entropy"] is not None:
            d -= s["d_entropy"][a:b, None].double() * (p * logp + p)
        return {"dlogits": (d - p * d.sum(1, keepdim=True)) / t}
    token, value, w = s["teacher_token"][a:b], s["teacher_value"][a:b].double(), s["weight"][a:b, None].double()
    on = torch.zeros_like(p).scatter_(1, token, 1.0)
    q = torch.softmax(value / t, 1) if case["teacher"] == "logits" else value.exp()
    loss = (torch.special.xlogy(q, q) - q * logp.gather(1, token)).sum(1, keepdim=True)
    d = torch.zeros_like(p).scatter_(1, token, -q)
    mass = q.sum(1, keepdim=True)
    if case["teacher"] == "logprobs":
        q_rest = (1.0 - mass).clamp(min=0.0)
        p_rest = (p * (1.0 - on)).sum(1, keepdim=True)
        loss = loss + torch.special.xlogy(q_rest, q_rest) - torch.special.xlogy(q_rest, p_rest)
        d = d - (1.0 - on) * p * (q_rest / p_rest)
        mass = mass + q_rest
    out = {"loss": torch.where(w != 0, loss, 0.0)[:, 0]}
    if case["grad"]:
        out["dlogits"] = (d + mass * p) * (w / t)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    block = max(1, (1 << 26) // case["vocab"])
    parts = [_exact_rows(s, a, min(case["rows"], a + block)) for a in range(0, case["rows"], block)]
    out = {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
    if case["op"] == "logprobs" and case["k"]:
        out["top_token"] = None
    return out
