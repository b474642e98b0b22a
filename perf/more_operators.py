"""Cases for a Worker's objectives on its own answers (clipped policy loss from the logits, preference loss from paired log
ratios) and for its step (AdamW over many tensors, with states in 32 bits or in 8).

``run`` computes a case either in plain torch operations (32 bits, one rounding at the end) or, where ``own`` is
true, through the library's entry points; ``exact`` gives the same outputs from the definitions in 64 bits.
"""
import math
import random

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
_BLOCK = 32  # elements that share a scale, where states are held in 8 bits


def _policy(name, rows, vocab, dtype, temperature=1.0, skip=0, kl=0.05, entropy=0.0, dual=0.0, grad=True, pad=0):
    return {"name": name, "op": "policy", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature, "skip": skip,
            "kl": kl, "entropy": entropy, "dual": dual, "grad": grad, "pad": pad}


def _preference(name, pairs, longest, ref, kind, normalise=False, smoothing=0.0, split=False):
    return {"name": name, "op": "preference", "pairs": pairs, "longest": longest, "ref": ref, "kind": kind,
            "normalise": normalise, "smoothing": smoothing, "split": split}


def _adam(name, n, tensors, param, grad, bits, master=False, clip=True, packed=False):
    return {"name": name, "op": "adam", "n": n, "tensors": tensors, "param": param, "grad": grad, "bits": bits,
            "master": master, "clip": clip, "packed": packed}


def listed():
    return [
        # one short answer in fp32, an odd vocabulary: latency
        _policy("policy_one_answer", 61, 20011, "f32", 0.7, entropy=0.01),
        # a policy step over a batch of answers, with the KL term to a reference
        _policy("policy_step", 4096, 131072, "bf16"),
        # ragged answers packed into a batch (an eighth of the rows are prompts or padding), odd vocabulary, entropy bonus, and
        # a second bound for answers that were worse than expected
        _policy("policy_ragged_odd", 2047, 100003, "bf16", skip=8, entropy=0.003, dual=3.0),
        # a few short pairs: latency
        _preference("preference_small", 4, 64, "f32", "logistic"),
        # a training step's batch of pairs with their prompts, chosen and rejected halves one after the other
        _preference("preference_batch", 1024, 2048, "f32", "logistic", smoothing=0.1, split=True),
        # few pairs of very long answers, mean log ratios, the reference's log probabilities stored in bf16
        _preference("preference_long", 12, 131072, "bf16", "squared", normalise=True),
        # a small network's tensors, as one parameter vector without gaps (no tensor but the first is aligned)
        _adam("adam_small_packed", 120_011, 14, "f32", "f32", 32, packed=True),
        # an image network's 25.6 million parameters in fp32
        _adam("adam_f32", 25_600_000, 161, "f32", "f32", 32, clip=False),
        # a language model's step in mixed precision: bf16 parameters and gradients, fp32 master copy, gradients clipped
        _adam("adam_bf16_master", 1 << 28, 291, "bf16", "bf16", 32, master=True),
        # states in 8 bits: a small network, and the same as one vector without gaps
        _adam("adam8_small", 400_000, 14, "f32", "f32", 8, clip=False),
        _adam("adam8_packed", 25_600_000, 161, "f32", "bf16", 8, packed=True),
        # a language model with bf16 parameters alone, rounded stochastically, gradients clipped: the largest
        _adam("adam8_bf16", 1 << 28, 291, "bf16", "bf16", 8),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "preference", "adam", "adam"])
    if op == "policy":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        vocab = _log_uniform(rng, 512, 262144)
        if rng.random() < 0.5:
            vocab = max(512, vocab // 128 * 128)
        rows = min(_log_uniform(rng, 1, 8192), (1 << 30) // _BYTES[dtype] // vocab)
        case = _policy("", rows, vocab, dtype, rng.choice([1.0, 1.0, 0.7]), rng.choice([0, 0, 4, 8]), rng.choice([0.0, 0.05]),
                       rng.choice([0.0, 0.01]), rng.choice([0.0, 3.0]), rng.random() < 0.8,
                       rng.choice([0, 0, 8, rng.randrange(1, 64)]))
    elif op == "preference":
        longest = _log_uniform(rng, 4, 131072)
        pairs = min(_log_uniform(rng, 1, 4096), (1 << 21) // longest + 1)
        case = _preference("", pairs, longest, rng.choice(["none", "f32", "bf16"]), rng.choice(["logistic", "hinge", "squared"]),
                           rng.random() < 0.5, rng.choice([0.0, 0.1]), rng.random() < 0.5)
    else:
        n = _log_uniform(rng, 2000, 1 << 27)
        param = rng.choice(["f32", "bf16"])
        case = _adam("", n, min(_log_uniform(rng, 1, 400), n // 500), param, rng.choice(["f32", "bf16"]), rng.choice([32, 8]),
                     param == "bf16" and rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.4)
    del case["name"]
    return case


def _kept_rows(case):
    """Rows that count: with ``skip`` = s every s-th row is padding."""
    return case["rows"] - (case["rows"] // case["skip"] if case["skip"] else 0)


def _lengths(case):
    """Prompt and answer lengths of a case's sequences, ragged, the longest as long as the case says."""
    rng = random.Random(case["pairs"] * 1_000_003 + case["longest"])
    longest = case["longest"]
    prompts, answers = [], []
    for s in range(2 * case["pairs"]):
        length = longest if s == 0 else rng.randrange(max(1, longest // 8), longest + 1)
        prompts.append(rng.randrange(0, length // 2 + 1))
        answers.append(length - prompts[-1])
    return prompts, answers


def _sizes(case):
    """Numbers of elements of a case's tensors: half of them small (gains, biases), the others share what is left."""
    n, count = case["n"], case["tensors"]
    rng = random.Random(n * 1_000_003 + count)
    small = [rng.randrange(1, max(2, min(8192, n // (2 * count)))) for _ in range(count // 2)]
    share = [math.exp(rng.uniform(0.0, 3.0)) for _ in range(count - len(small))]
    left, total = n - sum(small), sum(share)
    large = [max(1, int(left * w / total)) for w in share]
    large[0] += left - sum(large)
    sizes = small + large
    rng.shuffle(sizes)
    return sizes


def _blocks(sizes):
    return [(size + _BLOCK - 1) // _BLOCK for size in sizes]


def work(case):
    if case["op"] == "policy":
        rows, vocab, size = case["rows"], case["vocab"], _BYTES[case["dtype"]]
        kept = _kept_rows(case)
        # token, old and reference log probability, advantage and weight in; loss, log probability and entropy out
        small = rows * (8 + 4 + 4 + (4 if case["kl"] else 0) + 4 + 8 + (4 if case["entropy"] else 0))
        out = rows * vocab * size if case["grad"] else 0
        flops = 5 + (2 if case["entropy"] else 0) + (3 if case["grad"] else 0)
        return {"bytes": kept * vocab * size + out + small, "flops": flops * kept * vocab}
    if case["op"] == "preference":
        prompts, answers = _lengths(case)
        tokens = sum(prompts) + sum(answers)
        ref = {"none": 0, "f32": 4, "bf16": 2}[case["ref"]]
        return {"bytes": tokens * (8 + ref + 4) + case["pairs"] * 32, "flops": 4 * tokens}
    sizes = _sizes(case)
    n, blocks = sum(sizes), sum(_blocks(sizes))
    each = 2 * _BYTES[case["param"]] + _BYTES[case["grad"]] + (8 if case["master"] else 0)
    if case["bits"] == 8:  # read and written, with their scales; and written out as the values that they stand for
        return {"bytes": n * (each + 4) + 4 * blocks + 4 * _BLOCK * blocks, "flops": 30 * n}
    return {"bytes": n * (each + 16), "flops": (17 if case["clip"] else 14) * n}


# ---- inputs --------------------------------------------------------------------------------------------------------


def _prepare_policy(case, gen):
    rows, vocab, dtype, t = case["rows"], case["vocab"], _DTYPES[case["dtype"]], case["temperature"]
    order = torch.randperm(vocab, generator=gen, device="cuda")
    store = torch.empty((rows, vocab + case["pad"]), dtype=dtype, device="cuda")
    store.normal_(0.0, 2.5, generator=gen)  # a spread of a few units around a falling unigram prior
    store[:, :vocab] += (-0.8 * torch.log1p(order.float())).to(dtype)
    logits = store[:, :vocab]
    s = {"case": case, "logits": logits, "tokens": torch.empty(rows, dtype=torch.int64, device="cuda")}
    logprob = torch.empty(rows, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 512):  # tokens drawn from the model's own distribution, by blocks of rows
        z = logits[a:a + 512].double() / t
        noise = torch.empty_like(z).exponential_(1.0, generator=gen)
        s["tokens"][a:a + 512] = (z - noise.log()).argmax(1)
        logprob[a:a + 512] = z.gather(1, s["tokens"][a:a + 512, None])[:, 0] - torch.logsumexp(z, 1)
    # the policy that drew the answers is some steps older than the one that is trained: ratios around 1, a sixth of them
    # clipped.  Where a ratio meets a bound the gradient jumps, so none lies within 1e-3 of one.
    change = 0.15 * torch.randn(rows, generator=gen, device="cuda", dtype=torch.float64)
    for bound in (0.8, 1.2, 3.0):
        change = torch.where((change - math.log(bound)).abs() < 1e-3, change + 2e-3, change)
    s["old_logprob"] = (logprob - change).float()
    s["ref_logprob"] = (logprob + 0.3 * torch.randn(rows, generator=gen, device="cuda")).float() if case["kl"] else None
    s["advantage"] = torch.randn(rows, generator=gen, device="cuda")
    s["weight"] = torch.full((rows,), 1.0 / _kept_rows(case), device="cuda")
    if case["skip"]:
        s["weight"][case["skip"] - 1::case["skip"]] = 0.0
    s["loss"], s["logprob"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    s["entropy"] = torch.empty(rows, device="cuda") if case["entropy"] else None
    s["dlogits"] = torch.empty((rows, vocab), dtype=dtype, device="cuda") if case["grad"] else None
    return s


def _prepare_preference(case, gen):
    prompts, answers = _lengths(case)
    pairs = case["pairs"]
    lengths = torch.tensor([a + b for a, b in zip(prompts, answers)], dtype=torch.int64)
    prompt = torch.tensor(prompts, dtype=torch.int64)
    offsets = torch.zeros(2 * pairs + 1, dtype=torch.int64)
    offsets[1:] = torch.cumsum(lengths, 0)
    tokens = int(offsets[-1])
    s = {"case": case, "offsets": offsets.cuda()}
    sequence = torch.repeat_interleave(torch.arange(2 * pairs, device="cuda"), lengths.cuda())
    within = torch.arange(tokens, device="cuda") - s["offsets"][sequence]
    s["weight"] = (within >= prompt.cuda()[sequence]).float()  # prompts do not count
    # log probabilities of an answer's tokens: mostly likely ones, some rare
    ref = -torch.empty(tokens, device="cuda").exponential_(1.0, generator=gen)
    drift = torch.randn(2 * pairs, generator=gen, device="cuda") / lengths.cuda().float().sqrt()
    s["logprob"] = (ref + 0.1 * torch.randn(tokens, generator=gen, device="cuda") + drift[sequence]).clamp_(max=0.0)
    s["ref_logprob"] = None if case["ref"] == "none" else ref.to(_DTYPES[case["ref"]])
    s["pair_weight"] = torch.full((pairs,), 1.0 / pairs, device="cuda")
    # with a reference the log ratios are near 0; without one, means are compared with a margin
    s["beta"] = 2.0 if case["normalise"] else 0.1 if case["ref"] != "none" else 0.01
    s["margin"] = 0.5 if case["ref"] == "none" else 0.0
    s["loss"], s["reward"] = torch.empty(pairs, device="cuda"), torch.empty(2 * pairs, device="cuda")
    s["d_logprob"] = torch.empty(tokens, device="cuda")
    return s


_LR, _BETA1, _BETA2, _EPS, _DECAY, _MAX_NORM, _SEED = 3e-4, 0.9, 0.95, 1e-8, 0.1, 1.0, 20240917


def _prepare_adam(case, gen):
    sizes, count = _sizes(case), case["tensors"]
    blocks = _blocks(sizes)
    total = _BLOCK * sum(blocks)
    # where each tensor begins: in the vectors as they are stored, and in steps of whole blocks
    padded, packed = [0], [0]
    for size, block in zip(sizes, blocks):
        padded.append(padded[-1] + _BLOCK * block)
        packed.append(packed[-1] + size)
    begin = packed if case["packed"] else padded
    s = {"case": case, "steps": 1000, "step": torch.full((1,), 1000, dtype=torch.int64, device="cuda")}
    tensor = torch.repeat_interleave(torch.arange(count, device="cuda"), torch.tensor(blocks, device="cuda"))
    inside = torch.arange(total, device="cuda", dtype=torch.int32)
    size_of, begin_of = torch.tensor(sizes, device="cuda"), torch.tensor(padded[:-1], device="cuda")
    inside = (inside.view(-1, _BLOCK) - begin_of[tensor, None].int()) < size_of[tensor, None].int()
    inside = inside.view(-1)
    if case["packed"]:  # place of each stored element in whole blocks
        s["place"] = inside.nonzero()[:, 0]
    decay = torch.tensor([0.0 if size <= 8192 else _DECAY for size in sizes], dtype=torch.float64)
    s["decay"] = decay.cuda()[tensor]
    spread = (1e-3 * torch.exp(2.0 * torch.randn(count, generator=gen, device="cuda")))[tensor]

    def of_blocks(x, dtype=torch.float32):  # from whole blocks to what is stored
        x = (x * inside).to(dtype)
        return x[s["place"]].contiguous() if case["packed"] else x

    def noise():
        return torch.randn(total, generator=gen, device="cuda")

    def scaled(x):
        return (x.view(-1, _BLOCK) * spread[:, None]).view(-1)

    s["theta"] = of_blocks(0.02 * noise(), _DTYPES[case["param"]])
    s["master"] = s["theta"].float() if case["master"] else None
    s["grad"] = of_blocks(scaled(noise()), _DTYPES[case["grad"]])
    m = scaled(0.3 * noise())
    root = scaled((noise().abs() + 0.2))
    if case["bits"] == 8:
        m, root = m * inside, root * inside
        s["m_scale"], s["v_scale"] = _scales(m), _scales(root)
        half = torch.full((total,), 1 << 15, device="cuda", dtype=torch.int32)  # to the nearest
        s["m"] = of_blocks(_to_codes(m, s["m_scale"], half, 3), torch.uint8)
        s["v"] = of_blocks(_to_codes(root, s["v_scale"], half, 4), torch.uint8)
        s["m_value"], s["root_value"] = (torch.empty(total, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    else:
        s["m_scale"] = s["v_scale"] = None
        s["m"], s["v"] = of_blocks(m), of_blocks(root * root)
    s["total"] = total
    s["sumsq"] = torch.zeros(1, dtype=torch.float64, device="cuda")
    s["plan"] = None
    if own:
        def tensors(x):
            return None if x is None else [x[a:a + size] for a, size in zip(begin, sizes)]

        def scale_tensors(x):
            return None if x is None else [x[a // _BLOCK:a // _BLOCK + b] for a, b in zip(padded, blocks)]

        s["plan"] = _qn().qn_adam_create(tensors(s["theta"]), tensors(s["grad"]), tensors(s["m"]), tensors(s["v"]),
                                         master=tensors(s["master"]), m_scale=scale_tensors(s["m_scale"]),
                                         v_scale=scale_tensors(s["v_scale"]), weight_decay=decay.tolist())
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    return {"policy": _prepare_policy, "preference": _prepare_preference, "adam": _prepare_adam}[case["op"]](case, gen)


# ---- plain forms ---------------------------------------------------------------------------------------------------

_CLIP = 0.2


def _plain_policy(s):
    case, w, advantage = s["case"], s["weight"], s["advantage"]
    u = s["logits"].float() / case["temperature"]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    total = e.sum(1, keepdim=True)
    shift = torch.log(total)
    logprob = (u.gather(1, s["tokens"][:, None]) - shift)[:, 0]
    ratio = torch.exp(logprob - s["old_logprob"])
    free, held = -advantage * ratio, -advantage * ratio.clamp(1.0 - _CLIP, 1.0 + _CLIP)
    loss, slope = torch.maximum(free, held), torch.where(free >= held, free, 0.0)
    if case["dual"]:
        most = -advantage * case["dual"]
        beyond = (advantage < 0) & (loss > most)
        loss, slope = torch.where(beyond, most, loss), torch.where(beyond, 0.0, slope)
    if case["kl"]:
        x = s["ref_logprob"] - logprob
        loss, slope = loss + case["kl"] * (torch.expm1(x) - x), slope - case["kl"] * torch.expm1(x)
    out = {"logprob": torch.where(w != 0, logprob, 0.0)}
    if case["entropy"]:
        entropy = (shift - (e * u).sum(1, keepdim=True) / total)[:, 0]
        loss = loss - case["entropy"] * entropy
        out["entropy"] = torch.where(w != 0, entropy, 0.0)
    out["loss"] = torch.where(w != 0, loss, 0.0)
    if case["grad"]:
        p = e / total
        d = p * -slope[:, None]
        if case["entropy"]:
            d = d + case["entropy"] * p * (u - shift + entropy[:, None])
        d.scatter_add_(1, s["tokens"][:, None], slope[:, None])
        out["dlogits"] = (d * (w / case["temperature"])[:, None]).to(s["logits"].dtype)
    return out


def _plain_preference(s):
    case, offsets, w = s["case"], s["offsets"], s["weight"].double()
    pairs, beta = case["pairs"], s["beta"]
    sequence = torch.repeat_interleave(torch.arange(2 * pairs, device="cuda"), offsets[1:] - offsets[:-1],
                                       output_size=s["logprob"].numel())
    ratio = s["logprob"].double()
    if s["ref_logprob"] is not None:
        ratio = ratio - s["ref_logprob"].double()
    zero = torch.zeros(1, dtype=torch.float64, device="cuda")
    sums = torch.cat([zero, (w * ratio).cumsum(0)])[offsets].diff()  # differences of running sums
    each = torch.full_like(sums, beta)
    if case["normalise"]:
        count = torch.cat([zero, w.cumsum(0)])[offsets].diff()
        each = torch.where(count > 0, beta / count, 0.0)
    reward = sums * each
    chosen = torch.arange(pairs, device="cuda") * (1 if case["split"] else 2)
    rejected = chosen + (pairs if case["split"] else 1)
    h = reward[chosen] - reward[rejected] - s["margin"]
    if case["kind"] == "logistic":
        keep = 1.0 - case["smoothing"]
        low = torch.log1p(torch.exp(-h.abs()))
        loss = keep * (low + (-h).clamp(min=0.0)) + case["smoothing"] * (low + h.clamp(min=0.0))
        slope = 1.0 / (1.0 + torch.exp(-h)) - keep
    elif case["kind"] == "hinge":
        loss, slope = (1.0 - h).clamp(min=0.0), -(h < 1.0).double()
    else:
        loss, slope = ((h - 0.5) / beta) ** 2, 2.0 * (h - 0.5) / beta ** 2
    slope = slope * s["pair_weight"]
    by_sequence = torch.empty_like(sums)
    by_sequence[chosen], by_sequence[rejected] = slope, -slope
    return {"loss": loss.float(), "reward": reward.float(), "d_logprob": ((by_sequence * each)[sequence] * w).float()}


# States in 8 bits.  A block of 32 elements has one power of two, 2^(scale - 127), chosen so that its largest magnitude is in
# [128, 256) times that (scale 0: a block of zeros).  Magnitudes are held with an exponent of 4 bits and a fraction of 3 (the
# moving average m, with a sign) or 4 bits (the root of the moving average of squares), rounded up or down by chance.

_LOW = 0xFFFFFFFF


def _mix(x):
    x = x & _LOW
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & _LOW
    x = x ^ (x >> 13)
    x = (x * 0x3C6EF373) & _LOW
    return x ^ (x >> 16)


def _key(seed, step):
    """Of one step: a hash of both numbers' halves."""
    key = _mix(_mix(seed) + (seed >> 32))
    return _mix(_mix(key + ((step & _LOW) * 0x9E3779B1 & _LOW)) + (step >> 32))


def _words(key, total):
    """A hash of 32 bits for each element, from one for each eight."""
    eights = torch.arange(total // 8, device="cuda", dtype=torch.int64)
    x = _mix(eights * 0x9E3779B1 + key)
    y = (x[:, None] + torch.arange(8, device="cuda", dtype=torch.int64) * 0x9E3779B1) & _LOW
    y = ((y ^ (y >> 15)) * 0xA54FF53B) & _LOW
    return (y ^ (y >> 16)).view(-1)


def _scales(x):
    most = x.abs().view(-1, _BLOCK).amax(1)
    scale = ((most.view(torch.int32) >> 23) - 7).clamp(1, 247)
    return torch.where(most > 0, scale, 0).to(torch.uint8)


def _power(exponent):
    return (exponent << 23).view(torch.float32)


def _to_codes(x, scale, chance, fraction):
    """Codes for the magnitudes of x; ``chance`` in [0, 2^16)."""
    drop = 23 - fraction
    up = _power(torch.where(scale > 0, 254 - scale.int(), 127))
    y = (x.abs().view(-1, _BLOCK) * up[:, None]).view(-1)
    small = y < 2.0 ** -6
    bits = torch.where(small, y + 2.0 ** -6, y).view(torch.int32)
    bits = (bits + (chance << (drop - 16)) + (1 << (drop - 17))) >> drop
    code = bits - (120 << fraction) - torch.where(small, 1 << fraction, 0)
    if fraction == 3:
        return code | torch.where(x < 0, 128, 0)
    return torch.where(x > 0, code.clamp(min=1), code)


def _from_codes(code, scale, fraction):
    code = code.int()
    magnitude = code & 127 if fraction == 3 else code
    small = magnitude < (1 << fraction)
    bits = torch.where(small, magnitude + (1 << fraction), magnitude) + (120 << fraction)
    y = (bits << (23 - fraction)).view(torch.float32)
    y = torch.where(small, y - 2.0 ** -6, y)
    if fraction == 3:
        y = torch.where(code >= 128, -y, y)
    return (y.view(-1, _BLOCK) * _power(scale.int())[:, None]).view(-1)


def _plain_adam(s):
    case, place, total = s["case"], s.get("place"), s["total"]

    def whole(x, dtype=torch.float32):
        x = x.to(dtype)
        return x if place is None else torch.zeros(total, dtype=dtype, device="cuda").index_copy_(0, place, x)

    def put(to, x):
        to.copy_(x if place is None else x[place])

    step = s["steps"] + 1
    s["steps"] = step
    s["step"].add_(1)
    grad = whole(s["grad"])
    if case["clip"]:
        s["sumsq"] = s["grad"].double().square().sum().view(1)
        norm = s["sumsq"].sqrt()
        grad = grad * torch.where(norm > _MAX_NORM, _MAX_NORM / norm, 1.0).float()
    theta = whole(s["theta"] if s["master"] is None else s["master"])
    if case["bits"] == 8:
        m = _from_codes(whole(s["m"], torch.uint8), s["m_scale"], 3)
        root = _from_codes(whole(s["v"], torch.uint8), s["v_scale"], 4)
        v = root * root
    else:
        m, v = whole(s["m"]), whole(s["v"])
    m = m * _BETA1 + grad * (1.0 - _BETA1)
    v = v * _BETA2 + grad * grad * (1.0 - _BETA2)
    root = torch.sqrt(v)
    speed, spread = _LR / (1.0 - _BETA1 ** step), 1.0 / math.sqrt(1.0 - _BETA2 ** step)
    theta = (theta.view(-1, _BLOCK) * (1.0 - _LR * s["decay"]).float()[:, None]).view(-1)
    theta = theta - (m * speed) / (root * spread + _EPS)
    out = {"theta": s["theta"], "step": s["step"]}
    if case["clip"]:
        out["sumsq"] = s["sumsq"]
    by_chance = case["param"] == "bf16" and not case["master"]
    word = _words(_key(_SEED, step), total) if case["bits"] == 8 or by_chance else None
    if by_chance:
        bits = theta.view(torch.int32) + ((word * 0x3C6EF373 & _LOW) >> 16).int()
        put(s["theta"], (bits & -65536).view(torch.float32).to(torch.bfloat16))
    else:
        put(s["theta"], theta.to(s["theta"].dtype))
    if case["master"]:
        put(s["master"], theta)
        out["master"] = s["master"]
    if case["bits"] == 8:
        s["m_scale"].copy_(_scales(m))
        s["v_scale"].copy_(_scales(root))
        m = _to_codes(m, s["m_scale"], (word >> 16).int(), 3)
        root = _to_codes(root, s["v_scale"], (word & 65535).int(), 4)
        put(s["m"], m.to(torch.uint8))
        put(s["v"], root.to(torch.uint8))
        s["m_value"].copy_(_from_codes(m, s["m_scale"], 3))
        s["root_value"].copy_(_from_codes(root, s["v_scale"], 4))
        out["m"], out["root"] = s["m_value"], s["root_value"]
    else:
        put(s["m"], m)
        put(s["v"], v)
        out["m"], out["v"] = s["m"], s["v"]
    return out


# ---- the library's calls -------------------------------------------------------------------------------------------


def _own_policy(s):
    case = s["case"]
    _qn().qn_policy(s["logits"], s["tokens"], s["old_logprob"], s["advantage"], s["loss"], dlogits=s["dlogits"],
                    ref_logprob=s["ref_logprob"], weight=s["weight"], logprob=s["logprob"], entropy=s["entropy"], clip_low=_CLIP,
                    clip_high=_CLIP, dual=case["dual"], kl=case["kl"], entropy_bonus=case["entropy"],
                    temperature=case["temperature"])
    return {name: s[name] for name in ("logprob", "entropy", "loss", "dlogits") if s[name] is not None}


def _own_preference(s):
    qn, case = _qn(), s["case"]
    kind = {"logistic": qn.QN_PREFERENCE_LOGISTIC, "hinge": qn.QN_PREFERENCE_HINGE, "squared": qn.QN_PREFERENCE_SQUARED}
    qn.qn_preference(s["logprob"], s["offsets"], s["loss"], d_logprob=s["d_logprob"], ref_logprob=s["ref_logprob"],
                     weight=s["weight"], pair_weight=s["pair_weight"], reward=s["reward"], kind=kind[case["kind"]],
                     beta=s["beta"], margin=s["margin"], smoothing=case["smoothing"], normalise=case["normalise"],
                     split=case["split"])
    return {"loss": s["loss"], "reward": s["reward"], "d_logprob": s["d_logprob"]}


def _own_adam(s):
    qn, case = _qn(), s["case"]
    out = {"theta": s["theta"], "step": s["step"]}
    if case["clip"]:
        qn.qn_adam_norm(s["plan"], s["sumsq"])
        out["sumsq"] = s["sumsq"]
    qn.qn_adam_step(s["plan"], s["step"], lr=_LR, beta1=_BETA1, beta2=_BETA2, eps=_EPS,
                    sumsq=s["sumsq"] if case["clip"] else None, max_norm=_MAX_NORM if case["clip"] else 0.0,
                    stochastic=True, seed=_SEED)
    if case["master"]:
        out["master"] = s["master"]
    if case["bits"] == 8:
        qn.qn_adam_state(s["plan"], s["m_value"], s["root_value"])
        out["m"], out["root"] = s["m_value"], s["root_value"]
    else:
        out["m"], out["v"] = s["m"], s["v"]
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return (_own_policy if op == "policy" else _own_preference if op == "preference" else _own_adam)(state)
    return (_plain_policy if op == "policy" else _plain_preference if op == "preference" else _plain_adam)(state)


# ---- 64 bits -------------------------------------------------------------------------------------------------------


def _exact_policy_rows(s, a, b):
    """The outputs for rows a..b: log_softmax, then the chain rule through the loss as a function of ln p of the token."""
    case, t, w = s["case"], s["case"]["temperature"], s["weight"][a:b, None].double()
    logp = torch.log_softmax(s["logits"][a:b].double() / t, 1)
    p = logp.exp()
    token = s["tokens"][a:b, None]
    lp = logp.gather(1, token)
    advantage, r = s["advantage"][a:b, None].double(), (lp - s["old_logprob"][a:b, None].double()).exp()
    gain = torch.minimum(advantage * r, advantage * r.clamp(1.0 - _CLIP, 1.0 + _CLIP))
    moves = ((advantage > 0) & (r <= 1.0 + _CLIP)) | ((advantage < 0) & (r >= 1.0 - _CLIP))
    if case["dual"]:
        least = torch.where(advantage < 0, case["dual"] * advantage, -math.inf)
        moves &= gain >= least
        gain = torch.maximum(gain, least)
    loss, slope = -gain, torch.where(moves, -advantage * r, 0.0)
    if case["kl"]:
        y = s["ref_logprob"][a:b, None].double() - lp
        loss = loss + case["kl"] * (y.exp() - 1.0 - y)
        slope = slope + case["kl"] * (1.0 - y.exp())
    entropy = torch.special.entr(p).sum(1, keepdim=True)
    loss = loss - case["entropy"] * entropy
    out = {"logprob": torch.where(w != 0, lp, 0.0)[:, 0], "loss": torch.where(w != 0, loss, 0.0)[:, 0]}
    if case["entropy"]:
        out["entropy"] = torch.where(w != 0, entropy, 0.0)[:, 0]
    if case["grad"]:
        d = torch.zeros_like(p).scatter_(1, token, slope) + case["entropy"] * p * (logp + 1.0)
        out["dlogits"] = (d - p * d.sum(1, keepdim=True)) * (w / t)
    return out


def _exact_preference(s):
    case, pairs, offsets = s["case"], s["case"]["pairs"], s["offsets"]
    w, ratio = s["weight"].double(), s["logprob"].double()
    if s["ref_logprob"] is not None:
        ratio = ratio - s["ref_logprob"].double()

    lengths = offsets[1:] - offsets[:-1]
    sequence = torch.repeat_interleave(torch.arange(2 * pairs, device="cuda"), lengths)

    def sums(x):
        return torch.zeros(2 * pairs, dtype=torch.float64, device="cuda").index_add_(0, sequence, x)

    count = sums(w) if case["normalise"] else torch.ones(2 * pairs, dtype=torch.float64, device="cuda")
    reward = torch.where(count > 0, s["beta"] * sums(w * ratio) / count, 0.0)
    split = reward.view(2, pairs) if case["split"] else reward.view(pairs, 2).t()
    h = (split[0] - split[1] - s["margin"]).requires_grad_()
    if case["kind"] == "logistic":
        loss = torch.logaddexp(-h, torch.zeros_like(h)) * (1.0 - case["smoothing"]) \
            + torch.logaddexp(h, torch.zeros_like(h)) * case["smoothing"]
    elif case["kind"] == "hinge":
        loss = torch.relu(1.0 - h)
    else:
        loss = (h / s["beta"] - 1.0 / (2.0 * s["beta"])) ** 2
    slope = torch.autograd.grad(loss, h, s["pair_weight"].double())[0]
    slope = torch.cat([slope, -slope]) if case["split"] else torch.stack([slope, -slope], 1).view(-1)
    each = torch.where(count > 0, s["beta"] * slope / count, 0.0)
    return {"loss": loss.detach(), "reward": reward, "d_logprob": each[sequence] * w}


def _round32(x):
    return x.float().double()


def _exact_codes(x, chance, bits):
    """The values that blocks x (in 64 bits, of numbers with 24) stand for once held in 8 bits, by the sizes of the steps."""
    most = x.abs().amax(1, keepdim=True)
    power = torch.where(most > 0, torch.frexp(most).exponent - 8, 0).clamp(min=-126)  # most / 2^power is in [128, 256)
    y = torch.ldexp(x.abs(), -power)
    low = 2.0 ** -6
    y = torch.where(y < low, _round32(y + low) - low, y)
    step = torch.ldexp(torch.ones_like(y), (torch.frexp(y).exponent - 1).clamp(min=-6) - bits)
    held = torch.floor(y / step + (chance + 0.5) / 65536.0) * step
    if bits == 4:
        held = torch.where(x > 0, torch.maximum(held, step.amin()), held)
    return torch.ldexp(held, power) * torch.sign(x)


def _exact_adam(s):
    """One step.  The states in 8 bits are defined from the moving averages in 32 bits, each operation rounded by itself."""
    case, total, place = s["case"], s["total"], s.get("place")
    step, f = s["steps"] + 1, (lambda x: torch.tensor(x, dtype=torch.float32).double().item())
    grad_all = s["grad"].double()
    sumsq, coefficient = grad_all.square().sum().view(1), 1.0
    if case["clip"]:
        coefficient = min(1.0, _MAX_NORM / math.sqrt(sumsq.item()))
    del grad_all
    if place is None:
        place = torch.arange(total, device="cuda")
    where = torch.full((total,), -1, dtype=torch.int64, device="cuda")
    where[place] = torch.arange(place.numel(), device="cuda")
    words = _words(_key(_SEED, step), total) if case["bits"] == 8 or case["param"] == "bf16" else None
    out = {name: [] for name in ("theta", "master", "m", "v", "root")}
    for a in range(0, total, 1 << 24):
        b = min(total, a + (1 << 24))
        at, here = where[a:b].clamp(min=0), where[a:b] >= 0

        def whole(x):
            return torch.where(here, x[at].double(), 0.0)

        def keep(name, x):
            out[name].append(x[here])

        decay = s["decay"][a // _BLOCK:b // _BLOCK].repeat_interleave(_BLOCK)
        theta, g = whole(s["theta"] if s["master"] is None else s["master"]), whole(s["grad"])
        if case["bits"] == 8:
            blocks = slice(a // _BLOCK, b // _BLOCK)
            g = _round32(g * f(coefficient))
            code, scale = whole(s["m"]), s["m_scale"][blocks].double().repeat_interleave(_BLOCK)
            sign, code = torch.where(code >= 128, -1.0, 1.0), code % 128
            m = sign * torch.where(code < 8, code / 8, 1 + code % 8 / 8) * 2.0 ** ((code // 8).clamp(min=1) - 7 + scale - 127)
            code, scale = whole(s["v"]), s["v_scale"][blocks].double().repeat_interleave(_BLOCK)
            r = torch.where(code < 16, code / 16, 1 + code % 16 / 16) * 2.0 ** ((code // 16).clamp(min=1) - 7 + scale - 127)
            m = _round32(_round32(m * f(_BETA1)) + _round32(g * f(1.0 - _BETA1)))
            v = _round32(_round32(_round32(r * r) * f(_BETA2)) + _round32(_round32(g * g) * f(1.0 - _BETA2)))
            root = _round32(torch.sqrt(v))
            out["m"].append(_exact_codes(m.view(-1, _BLOCK), (words[a:b] >> 16).double().view(-1, _BLOCK), 3).view(-1).bfloat16())
            out["root"].append(_exact_codes(root.view(-1, _BLOCK), (words[a:b] & 65535).double().view(-1, _BLOCK), 4).view(-1).bfloat16())
        else:
            g = g * coefficient
            m = _BETA1 * whole(s["m"]) + (1.0 - _BETA1) * g
            v = _BETA2 * whole(s["v"]) + (1.0 - _BETA2) * g * g
            root = torch.sqrt(v)
            keep("m", m)
            keep("v", v)
        step_size = m / (1.0 - _BETA1 ** step) / (root / math.sqrt(1.0 - _BETA2 ** step) + _EPS)
        theta = theta * (1.0 - _LR * decay) - _LR * step_size
        if case["master"]:
            keep("master", theta)
        elif case["param"] == "bf16":  # up or down by chance, in steps of 2^-7 of the power of two below
            unit = torch.ldexp(torch.ones_like(theta), torch.frexp(theta).exponent - 8)
            chance = ((words[a:b] * 0x3C6EF373 & _LOW) >> 16).double() / 65536.0
            theta = torch.sign(theta) * torch.floor(theta.abs() / unit + chance) * unit
        keep("theta", theta)
    out = {name: torch.cat(parts) for name, parts in out.items() if parts}
    out["step"] = s["step"] + 1
    if case["clip"]:
        out["sumsq"] = sumsq
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "preference":
        return _exact_preference(s)
    if case["op"] == "adam":
        return _exact_adam(s)
    block = max(1, (1 << 26) // case["vocab"])
    parts = [_exact_policy_rows(s, a, min(case["rows"], a + block)) for a in range(0, case["rows"], block)]
    return {name: torch.cat([part[name] for part in parts]) for name in parts[0]}
