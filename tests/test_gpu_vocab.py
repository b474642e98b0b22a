"""The operators over a vocabulary (qn_logprobs, qn_logprobs_backward, qn_distill) against plain 64-bit forms.

Tolerances.  A sum of positive fp32 terms by threads (at most a few thousand each) and then over the row is off by
about sqrt(terms) * 6e-8 < 4e-6 of itself, exp2 by 2.4e-7, a logarithm near 20 by 1e-6: 5e-6 (1 + |value|) for numbers
per row, 1e-5 of the summed magnitudes of its terms for an element of a gradient, and for bf16 storage one rounding
(2^-9, taken as 2^-8) on top.
"""
import math

import pytest
import torch

import vocab_reference as ref

pytestmark = pytest.mark.gpu

INF = math.inf
DTYPES = [torch.float32, torch.bfloat16]
PATTERN = {torch.float32: -7.25, torch.bfloat16: -7.25, torch.int64: -77}


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import qn as mod

    assert torch.cuda.is_available()
    mod.lib()
    return mod


class Out:
    """Contiguous outputs inside guard bands: ``check`` fails if a kernel wrote outside of them."""

    def __init__(self):
        self.kept = []

    def new(self, shape, dtype, stride=None, offset=0):
        rows = shape[0]
        step = stride or (math.prod(shape[1:]) if len(shape) > 1 else 1)
        n = 64 + offset + rows * step + 64
        full = torch.full((n,), PATTERN[dtype], dtype=dtype, device="cuda")
        view = full.as_strided(shape, (step, 1) if len(shape) == 2 else (1,), 64 + offset)
        self.kept.append((full, view, dtype))
        return view

    def check(self):
        for full, view, dtype in self.kept:
            mask = torch.ones_like(full, dtype=torch.bool)
            mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
            assert bool((full[mask] == PATTERN[dtype]).all()), "write outside an output"


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    same = (got == want) | (got.isnan() & want.isnan())
    ok = same | ((got - want).abs() <= bound)
    assert bool(ok.all()), (what, got[~ok][:8], want[~ok][:8], bound.expand_as(got)[~ok][:8])


def run_logprobs(qn, z, tokens, k, temperature=1.0, stream=None):
    rows = z.shape[0]
    o = Out()
    lp, lse, ent = (o.new((rows,), torch.float32) for _ in range(3))
    top = o.new((rows, k), torch.int64) if k else None
    top_lp = o.new((rows, k), torch.float32) if k else None
    qn.qn_logprobs(z, tokens, lp, lse=lse, entropy=ent, top_token=top, top_logprob=top_lp, temperature=temperature,
                   stream=stream)
    return o, lp, lse, ent, top, top_lp


def check_logprobs(qn, z, tokens, k, temperature=1.0):
    o, lp, lse, ent, top, top_lp = run_logprobs(qn, z, tokens, k, temperature)
    want = ref.logprobs64(z, tokens, k, temperature)
    torch.cuda.synchronize()
    o.check()

    def bound(x):
        return 5e-6 * (1 + x.abs().nan_to_num(0, 0, 0))

    # logprob and the alternatives are differences from the row's largest logit, which may be large
    close(lp, want[0], bound(want[0]), "logprob")
    close(lse, want[1], bound(want[1]), "lse")
    close(ent, want[2], bound(want[2]), "entropy")
    if k:
        assert torch.equal(top, want[3]), (top[(top != want[3]).any(1)][:2], want[3][(top != want[3]).any(1)][:2])
        close(top_lp, want[4], bound(want[4]), "top_logprob")
    return lp, lse, ent, top, top_lp


def some_tokens(rows, vocab, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t[::5] = -100
    return t


SHAPES = [(1, 1), (3, 1), (1, 2), (2, 3), (5, 7), (4, 8), (3, 9), (1, 31), (7, 33), (2, 255), (300, 257), (3, 1000),
          (17, 4097), (2, 8192), (5, 16389), (1, 32768), (3, 50001), (2, 131072), (1, 262147)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_logprobs_shapes(qn, rows, vocab, dtype):
    z = ref.make_logits(rows, vocab, dtype, rows + vocab)
    check_logprobs(qn, z, some_tokens(rows, vocab, 1), min(5, vocab), 1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("k", [0, 1, 2, 20, 63, 64, 65, 128])
@pytest.mark.parametrize("rows,vocab", [(3, 40), (2, 1031), (400, 2048), (5, 33333), (1, 140000)])
def test_logprobs_alternatives(qn, rows, vocab, k, dtype):
    z = ref.make_logits(rows, vocab, dtype, k + vocab)  # bf16: many ties among the largest; k may exceed vocab
    check_logprobs(qn, z, some_tokens(rows, vocab, 2), k, 0.7)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (64, 2), (7, 7)])
def test_logprobs_strides(qn, dtype, pad, offset):
    for rows, vocab in ((9, 1003), (3, 20000), (2, 70001), (3, 5)):
        z = ref.make_logits(rows, vocab, dtype, pad, pad, offset)
        check_logprobs(qn, z, some_tokens(rows, vocab, 3), 5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [50, 1001, 40000, 200000])
def test_logprobs_masks(qn, vocab, dtype):
    """Rows with masked tokens, with nothing left, with one token left, of the type's lowest value, with NaN, with
    +inf, of extreme and of equal values: each has its own answer and none reaches its neighbour."""
    rows = 14
    z = ref.make_logits(rows, vocab, dtype, 11)
    tokens = torch.full((rows,), 7, device="cuda")
    low = torch.finfo(dtype).min
    z[1, ::2] = -INF
    z[2] = -INF
    z[3] = -INF
    z[3, vocab - 1] = 2.0
    z[4] = low
    z[5, 1::3] = low
    z[6, vocab // 2] = math.nan
    z[7, vocab - 2] = INF
    z[8] = 0.0
    z[9] = -0.0
    z[9, ::7] = 0.0
    z[10] = 1e30
    z[11, 3] = 3e38
    z[12] = torch.where(torch.arange(vocab, device="cuda") % 5 == 0, torch.finfo(dtype).min, -INF).to(dtype)
    z[13] = -INF
    z[13, 0] = math.nan
    tokens[3] = vocab - 1
    tokens[12] = 5
    tokens[8] = vocab  # not a token: NaN
    tokens[9] = -1
    for k in (0, 4, 40):
        lp, lse, ent, top, top_lp = check_logprobs(qn, z, tokens, k)
        assert lp[2] == -INF and lse[2] == -INF and ent[2] == 0 and lp[3] == 0 and ent[3] == 0
        assert lp[6].isnan() and lse[6].isnan() and lse[7].isnan() and lp[8].isnan() and lp[9] == 0
        assert abs(float(lp[4]) + math.log(vocab)) < 1e-4
        if k:
            assert int(top[3, 0]) == vocab - 1 and int(top[3, 1]) == -1 and int(top[2, 0]) == -1
            assert top[8].tolist() == list(range(k)) and top[9].tolist() == list(range(k))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kind", ["constant", "ascending", "descending", "two_values", "clustered", "periodic", "steps"])
def test_logprobs_adversarial_orders(qn, kind, dtype):
    """Orders and ties that make a selection of the largest values work hard."""
    rows, vocab = 3, 60007
    i = torch.arange(vocab, device="cuda", dtype=torch.float32)
    z = {"constant": torch.full_like(i, 1.5), "ascending": i / 1000, "descending": -i / 1000,
         "two_values": (i % 2), "clustered": torch.where((i > 30000) & (i < 31000), 5 + i / 1e4, -i / 1e5),
         # the large values a fixed distance apart, so that a few threads may hold all of them
         "periodic": torch.where(i % 2048 < 8, 10 + i / vocab, i / vocab), "steps": (i / 3000).floor()}[kind]
    z = z.to(dtype).expand(rows, vocab).contiguous()
    z[1] = z[1].flip(0)
    for k in (1, 64, 128):
        check_logprobs(qn, z, some_tokens(rows, vocab, 5), k)


def test_logprobs_partial_outputs(qn):
    z = ref.make_logits(6, 999, torch.bfloat16, 3)
    t = some_tokens(6, 999, 1)
    full = check_logprobs(qn, z, t, 3)
    for which in range(4):
        o = [torch.full((6,), 9.0, device="cuda") for _ in range(3)]
        top, top_lp = torch.zeros((6, 3), dtype=torch.int64, device="cuda"), torch.zeros((6, 3), device="cuda")
        if which < 3:
            args = [None, None, None]
            args[which] = o[which]
            qn.qn_logprobs(z, t if which == 0 else None, *args)
            assert torch.equal(o[which], full[which])
        else:
            qn.qn_logprobs(z, top_token=top, top_logprob=top_lp)
            assert torch.equal(top, full[3]) and torch.equal(top_lp, full[4])


def test_zero_rows_do_nothing(qn):
    for dtype in DTYPES:
        z = torch.empty((0, 100), dtype=dtype, device="cuda")
        v = torch.empty(0, device="cuda")
        t = torch.empty(0, dtype=torch.int64, device="cuda")
        qn.qn_logprobs(z, t, v)
        qn.qn_logprobs_backward(z, z.clone(), tokens=t, d_logprob=v)
        qn.qn_distill(z, t.view(0, 1).expand(0, 4).contiguous(), v.view(0, 1).expand(0, 4).contiguous(), v)


# ---- backward ------------------------------------------------------------------------------------------------------


def upstream(rows, seed, *more):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, *more), generator=gen, device="cuda")


def check_backward(qn, z, tokens, temperature, dlp, dl, dh, top, dt, pad=0, offset=0, inplace=False):
    rows, vocab = z.shape
    want, size = ref.backward64(z, tokens, temperature, dlp, dl, dh, top, dt)
    o = Out()
    if inplace:
        out = z.clone(memory_format=torch.preserve_format)
        src = out
    else:
        src, out = z, o.new((rows, vocab), z.dtype, vocab + pad, offset)
    qn.qn_logprobs_backward(src, out, tokens=tokens, d_logprob=dlp, d_lse=dl, d_entropy=dh, top_token=top,
                            d_top_logprob=dt, temperature=temperature)
    torch.cuda.synchronize()
    o.check()
    bound = 1e-5 * size + 1e-30
    if z.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * want.abs() + 2.0 ** -133
    close(out, want, bound, "dlogits")
    return out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_backward_shapes(qn, rows, vocab, dtype):
    z = ref.make_logits(rows, vocab, dtype, rows * 3 + vocab)
    t = some_tokens(rows, vocab, 4)
    check_backward(qn, z, t, 1.0, upstream(rows, 1), None, None, None, None)
    k = min(3, vocab)
    top = z.float().topk(k, 1).indices
    check_backward(qn, z, t, 0.7, upstream(rows, 1), upstream(rows, 2), upstream(rows, 3), top, upstream(rows, 4, k))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (64, 2)])
def test_backward_strides(qn, dtype, pad, offset):
    for rows, vocab in ((9, 1003), (2, 70001), (3, 5)):
        z = ref.make_logits(rows, vocab, dtype, pad, pad, offset)
        t = some_tokens(rows, vocab, 3)
        g = upstream(rows, 9)
        for out_pad, out_offset in ((pad, offset), (0, 0), (5, 3)):
            check_backward(qn, z, t, 1.0, g, None, -g, None, None, out_pad, out_offset)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [33, 5000, 150001])
def test_backward_in_place_repeats_and_padding(qn, vocab, dtype):
    """The gradient takes the logits' place; the given token also occurs among the alternatives, some alternatives are
    absent (-1) with a NaN gradient, and rows without upstream gradients hold NaN."""
    rows, k = 12, 9
    z = ref.make_logits(rows, vocab, dtype, 8)
    top = z.float().topk(k, 1).indices
    t = top[:, 2].clone()
    top[:, 4] = top[:, 5]  # twice the same
    top[3] = -1
    top[5, 7:] = -1
    g, gt = upstream(rows, 2), upstream(rows, 3, k)
    gt[5, 7:] = math.nan
    g[::4] = 0
    gt[::4] = 0
    t[1] = -5
    z[4] = math.nan
    z[8, 1:] = INF
    out = check_backward(qn, z, t, 1.3, g, None, None, top, gt)
    again = check_backward(qn, z, t, 1.3, g, None, None, top, gt, inplace=True)
    assert torch.equal(out.contiguous().view(torch.uint8), again.contiguous().view(torch.uint8))
    assert bool((out[4] == 0).all()) and bool((out[8] == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [64, 3001, 90000])
def test_backward_masks(qn, vocab, dtype):
    """Masked tokens, an empty row, rows of the type's lowest value and of large values (whose lse would have
    lost its logarithm to rounding), and a row without a distribution."""
    rows = 9
    z = ref.make_logits(rows, vocab, dtype, 21)
    low = torch.finfo(dtype).min
    z[1, ::2] = -INF
    z[2] = -INF
    z[3] = low
    z[4, 1::3] = low
    z[5] = 1e30
    z[6] += 3000.0
    z[7] -= 3000.0
    t = torch.full((rows,), 5, device="cuda")
    t[1] = 4  # masked
    g = upstream(rows, 5)
    for temperature in (1.0, 0.5):
        out = check_backward(qn, z, t, temperature, g, None, upstream(rows, 6), None, None)
        assert bool(torch.isfinite(out).all())
        assert bool((out[2].nonzero() == 5).all())
    z[8, 9] = math.nan
    out = torch.zeros_like(z)
    qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g)
    assert bool(out[8].isnan().all()) and bool(torch.isfinite(out[:8]).all())


def test_backward_against_differences(qn):
    """Against central differences of the 64-bit function, coordinate by coordinate."""
    rows, vocab, k, temperature = 2, 37, 4, 0.8
    z = ref.make_logits(rows, vocab, torch.float32, 77, spread=1.5)
    t = torch.tensor([3, 36], device="cuda")
    dlp, dl, dh, dt = upstream(rows, 1), upstream(rows, 2), upstream(rows, 3), upstream(rows, 4, k)
    lp, lse, ent, top, top_lp = check_logprobs(qn, z, t, k, temperature)
    out = torch.empty_like(z)
    qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=dlp, d_lse=dl, d_entropy=dh, top_token=top, d_top_logprob=dt,
                            temperature=temperature)

    def value(x):
        logp = torch.log_softmax(x / temperature, 1)
        h = -(logp.exp() * logp).sum(1)
        return (dlp * logp.gather(1, t[:, None])[:, 0] + dl * torch.logsumexp(x / temperature, 1) + dh * h
                + (dt * logp.gather(1, top)).sum(1))

    x, h = z.double(), 1e-5
    for i in range(vocab):
        e = torch.zeros_like(x)
        e[:, i] = h
        want = (value(x + e) - value(x - e)) / (2 * h)
        close(out[:, i], want, torch.full((1,), 2e-5, dtype=torch.float64, device="cuda"), i)


# ---- distillation --------------------------------------------------------------------------------------------------


def make_teacher(z, k, temperature, logprobs, seed, dtype=torch.float32):
    """A teacher near the student: its top k tokens and log probabilities, or logits."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = z.double().nan_to_num(0, 0, 0).clamp(-50, 50) + torch.randn(z.shape, generator=gen, device="cuda")
    top = t.topk(k, 1)
    value = (torch.log_softmax(t / temperature, 1).gather(1, top.indices) if logprobs else top.values)
    return top.indices, value.to(dtype)


def check_distill(qn, z, token, value, logprobs, temperature=1.0, weight=None, pad=0, offset=0, inplace=False):
    rows, vocab = z.shape
    want, grad, loss_size, size, slack = ref.distill64(z, token, value, logprobs, temperature, weight)
    mode = qn.QN_TEACHER_LOGPROBS if logprobs else qn.QN_TEACHER_LOGITS
    o = Out()
    loss, alone = o.new((rows,), torch.float32), o.new((rows,), torch.float32)
    if inplace:
        out = z.clone(memory_format=torch.preserve_format)
        src = out
    else:
        src, out = z, o.new((rows, vocab), z.dtype, vocab + pad, offset)
    qn.qn_distill(src, token, value, alone, weight=weight, temperature=temperature, teacher=mode)
    qn.qn_distill(src, token, value, loss, dlogits=out, weight=weight, temperature=temperature, teacher=mode)
    torch.cuda.synchronize()
    o.check()
    close(loss, want, 5e-6 * (1 + loss_size.nan_to_num(0, 0, 0)), "loss")
    assert torch.equal(loss.view(torch.int32), alone.view(torch.int32))
    bound = 1e-5 * size + 1e-6 * slack + 1e-30
    if z.dtype == torch.bfloat16:
        bound = bound + 2.0 ** -8 * grad.abs() + 2.0 ** -133
    close(out, grad, bound, "dlogits")
    return loss, out


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_distill_shapes(qn, rows, vocab, logprobs, dtype):
    z = ref.make_logits(rows, vocab, dtype, rows * 7 + vocab)
    k = min(6, vocab)  # for the smallest the list names the whole vocabulary
    token, value = make_teacher(z, k, 1.0, logprobs, 5)
    check_distill(qn, z, token, value, logprobs)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("k", [1, 2, 31, 33, 64, 100, 128])
def test_distill_lists(qn, k, logprobs, dtype):
    for rows, vocab in ((40, 300), (3, 30011), (2, 140001)):
        z = ref.make_logits(rows, vocab, dtype, k)
        token, value = make_teacher(z, k, 2.0, logprobs, k, torch.bfloat16 if k % 2 else torch.float32)
        w = upstream(rows, k)
        check_distill(qn, z, token, value, logprobs, 2.0, w)


def test_distill_largest_vocabulary(qn):
    for dtype in DTYPES:
        z = ref.make_logits(3, qn.QN_GRAD_MAX_VOCAB, dtype, 4, pad=3)
        token, value = make_teacher(z, 64, 1.0, True, 6)
        check_distill(qn, z, token, value, True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (8, 0), (64, 2)])
def test_distill_strides(qn, dtype, pad, offset):
    for rows, vocab in ((9, 1003), (2, 70001), (3, 5)):
        z = ref.make_logits(rows, vocab, dtype, pad, pad, offset)
        token, value = make_teacher(z, 4, 1.0, True, pad)
        for out_pad, out_offset in ((pad, offset), (0, 0), (5, 3)):
            check_distill(qn, z, token, value, True, 1.0, None, out_pad, out_offset)
        check_distill(qn, z, token, value, True, 1.0, None, inplace=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("vocab", [40, 3001, 90000])
def test_distill_masks(qn, vocab, logprobs, dtype):
    """Absent teacher tokens, rows without any, padding rows that hold NaN, masked logits on and off the list, rows of
    the type's lowest value and an empty row."""
    rows, k = 12, 7
    z = ref.make_logits(rows, vocab, dtype, 31)
    token, value = make_teacher(z, k, 1.0, logprobs, 3)
    w = torch.rand(rows, device="cuda") + 0.5
    token[0, 3:] = -1
    value[0, 3:] = math.nan  # not looked at
    token[1] = -1
    z[2] = math.nan
    w[2] = 0.0
    off = torch.ones((rows, vocab), dtype=torch.bool, device="cuda").scatter_(1, token.clamp(min=0), False)
    z[3] = torch.where(off[3] & (torch.arange(vocab, device="cuda") % 2 == 0), -INF, z[3].float()).to(dtype)
    z[4, token[4, 1]] = -INF  # the teacher wants what the student masks
    z[5] = torch.finfo(dtype).min
    z[6] = -INF
    value[7, 2] = -INF  # an entry that weighs nothing
    z[8] = torch.where(off[8], torch.finfo(dtype).min, z[8].float()).to(dtype) if not logprobs else z[8]
    token[9, 0], value[9, 0] = token[9, 1].clone(), value[9, 0]
    token[9, 0] = -1
    value[10] = -INF
    loss, out = check_distill(qn, z, token, value, logprobs, 1.0, w)
    assert loss[1] == 0 and loss[2] == 0 and loss[4] == INF and loss[6] == INF
    assert bool((out[1] == 0).all()) and bool((out[2] == 0).all()) and bool((out[6] == 0).all())
    assert bool(torch.isfinite(out).all())
    z[11, vocab // 3] = INF
    token[3, 2] = vocab  # no such token
    z[7, 1] = math.nan
    loss, out = torch.empty(rows, device="cuda"), torch.empty_like(z)
    qn.qn_distill(z, token, value, loss, dlogits=out, weight=w, teacher=qn.QN_TEACHER_LOGPROBS if logprobs else 0)
    for r in range(rows):
        assert bool(out[r].isnan().all() if r in (3, 7, 11) else torch.isfinite(out[r]).all()), r
        assert bool(loss[r].isnan()) == (r in (3, 7, 11)), r


def test_distill_repeated_token_stays_in_bounds(qn):
    z = ref.make_logits(4, 5003, torch.bfloat16, 2)
    token, value = make_teacher(z, 8, 1.0, True, 1)
    token[1] = token[1, 0].clone()
    o = Out()
    loss, out = o.new((4,), torch.float32), o.new((4, 5003), torch.bfloat16)
    qn.qn_distill(z, token, value, loss, dlogits=out)
    o.check()
    assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("logprobs", [False, True])
def test_distill_against_differences(qn, logprobs):
    """The gradient against central differences, of the 64-bit loss and of the kernel's own."""
    rows, vocab, k, temperature = 2, 41, 5, 1.7
    z = ref.make_logits(rows, vocab, torch.float32, 13, spread=1.5)
    token, value = make_teacher(z, k, temperature, logprobs, 2)
    loss, out = check_distill(qn, z, token, value, logprobs, temperature)
    mode = qn.QN_TEACHER_LOGPROBS if logprobs else qn.QN_TEACHER_LOGITS

    def mine(x):
        r = torch.empty(rows, device="cuda")
        qn.qn_distill(x, token, value, r, temperature=temperature, teacher=mode)
        return r.double()

    def theirs(x):
        return ref.distill64(x, token, value, logprobs, temperature, None)[0]

    for i in range(vocab):
        # third derivatives of L stay below 1 / T^3: h^2 / 6 and the noise 5e-6 (1 + sizes) / h bound the quotients
        for f, x, h, tol in ((theirs, z.double(), 1e-4, 2e-5), (mine, z, 2.0 ** -5, 2e-3)):
            e = torch.zeros_like(x)
            e[:, i] = h
            want = (f(x + e) - f(x - e)) / ((x + e) - (x - e))[:, i].double()
            close(out[:, i], want, torch.full((1,), tol, dtype=torch.float64, device="cuda"), i)


def test_teacher_to_student(qn):
    """What qn_logprobs writes of a teacher is what qn_distill takes: a student equal to its teacher has loss 0 and no
    gradient."""
    for dtype in DTYPES:
        for temperature in (1.0, 2.0):
            z = ref.make_logits(20, 9001, dtype, 3)
            top = torch.empty((20, 32), dtype=torch.int64, device="cuda")
            top_lp = torch.empty((20, 32), device="cuda")
            qn.qn_logprobs(z, top_token=top, top_logprob=top_lp, temperature=temperature)
            loss, out = check_distill(qn, z, top, top_lp, True, temperature)
            assert float(loss.abs().max()) < 1e-5 and float(out.float().abs().max()) < 1e-5


# ---- how the calls behave ------------------------------------------------------------------------------------------


def three_calls(qn, z, s, stream=None):
    qn.qn_logprobs(z, s["t"], s["lp"], lse=s["lse"], entropy=s["ent"], top_token=s["top"], top_logprob=s["top_lp"],
                   stream=stream)
    qn.qn_logprobs_backward(z, s["d1"], tokens=s["t"], d_logprob=s["g"], d_entropy=s["g"], stream=stream)
    qn.qn_distill(z, s["top"], s["top_lp"], s["loss"], dlogits=s["d2"], stream=stream)


def new_state(z, k=9):
    rows, vocab = z.shape
    f = {n: torch.zeros(rows, device="cuda") for n in ("lp", "lse", "ent", "loss")}
    return f | {"t": some_tokens(rows, vocab, 1), "g": upstream(rows, 1), "d1": torch.zeros_like(z),
                "d2": torch.zeros_like(z), "top": torch.zeros((rows, k), dtype=torch.int64, device="cuda"),
                "top_lp": torch.zeros((rows, k), device="cuda")}


def same(a, b):
    for n in a:
        assert torch.equal(a[n].contiguous().view(torch.uint8), b[n].contiguous().view(torch.uint8)), n


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(1, 100000), (200, 7001), (600, 32768), (3, 131072)])
def test_same_bits_each_time_on_any_stream_and_in_a_graph(qn, rows, vocab, dtype):
    z = ref.make_logits(rows, vocab, dtype, 6)
    a, b, c = new_state(z), new_state(z), new_state(z)
    three_calls(qn, z, a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    three_calls(qn, z, b, stream=side)
    side.synchronize()
    same(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        three_calls(qn, z, c)
    graph.replay()
    torch.cuda.synchronize()
    same(a, c)


def test_calls_on_two_streams_do_not_meet(qn):
    """No workspace: calls that overlap give what they give alone."""
    zs = [ref.make_logits(64, 30000 + 7 * i, torch.bfloat16, i) for i in range(2)]
    alone = [new_state(z) for z in zs]
    for z, s in zip(zs, alone):
        three_calls(qn, z, s)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in zs]
    both = [new_state(z) for z in zs]
    torch.cuda.synchronize()
    for _ in range(5):
        for z, s, st in zip(zs, both, streams):
            three_calls(qn, z, s, stream=st)
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        same(a, b)


def test_offsets_past_32_bits(qn):
    """Rows that start beyond 2^31 elements and 2^32 bytes."""
    stride, vocab = (1 << 31) + 24, 5000
    store = torch.zeros(2 * stride + vocab, dtype=torch.bfloat16, device="cuda")
    z = store.as_strided((3, vocab), (stride, 1))
    near = ref.make_logits(3, vocab, torch.bfloat16, 9)
    z.copy_(near)
    a, b = new_state(near), new_state(near)
    b["d1"] = b["d2"] = z  # the gradients in place, one after the other
    three_calls(qn, near, a)
    qn.qn_logprobs(z, b["t"], b["lp"], lse=b["lse"], entropy=b["ent"], top_token=b["top"], top_logprob=b["top_lp"])
    qn.qn_logprobs_backward(z, z, tokens=b["t"], d_logprob=b["g"], d_entropy=b["g"])
    assert torch.equal(z, a["d1"])
    z.copy_(near)
    qn.qn_distill(z, b["top"], b["top_lp"], b["loss"], dlogits=z)
    assert torch.equal(z, a["d2"])
    for n in ("lp", "lse", "ent", "loss", "top", "top_lp"):
        assert torch.equal(a[n], b[n]), n


def test_many_rows_of_one_vocabulary_entry(qn):
    """More rows than a grid dimension of 65535 would hold."""
    z = ref.make_logits(200_003, 3, torch.bfloat16, 1)
    check_logprobs(qn, z, some_tokens(200_003, 3, 1), 2)
    token, value = make_teacher(z, 2, 1.0, True, 1)
    check_distill(qn, z, token, value, True)


def test_refusals(qn):
    rows, vocab, k = 4, 100, 3
    z = torch.zeros((rows, vocab), device="cuda")
    t = torch.zeros(rows, dtype=torch.int64, device="cuda")
    f = [torch.zeros(rows, device="cuda") for _ in range(6)]
    top, top_lp = torch.zeros((rows, k), dtype=torch.int64, device="cuda"), torch.zeros((rows, k), device="cuda")
    out = torch.zeros_like(z)
    L, bad = qn.lib(), qn.QN_ERR_INVALID
    host = torch.zeros(rows * vocab * 4)

    def call(name, good, **change):
        args = dict(good, **change)
        return getattr(L, name)(*args.values())

    p = lambda x: x.data_ptr()  # noqa: E731
    fwd = {"rows": rows, "vocab": vocab, "dtype": 0, "logits": p(z), "stride": vocab, "tokens": p(t), "temperature": 1.0,
           "logprob": p(f[0]), "lse": p(f[1]), "entropy": p(f[2]), "k": k, "top": p(top), "top_lp": p(top_lp), "stream": 0}
    bwd = {"rows": rows, "vocab": vocab, "dtype": 0, "logits": p(z), "stride": vocab, "tokens": p(t), "temperature": 1.0,
           "dlp": p(f[3]), "dlse": p(f[4]), "dh": p(f[5]), "k": k, "top": p(top), "dtop": p(top_lp), "out": p(out),
           "out_stride": vocab, "stream": 0}
    dis = {"rows": rows, "vocab": vocab, "dtype": 0, "logits": p(z), "stride": vocab, "k": k, "token": p(top),
           "value_dtype": 0, "value": p(top_lp), "teacher": 1, "temperature": 1.0, "weight": p(f[0]), "loss": p(f[1]),
           "out": p(out), "out_stride": vocab, "stream": 0}
    common = [dict(rows=-1), dict(vocab=0), dict(vocab=1 << 31), dict(dtype=2), dict(dtype=-1), dict(logits=0),
              dict(logits=p(z) + 1), dict(logits=p(host)), dict(stride=vocab - 1), dict(temperature=0.0),
              dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=INF), dict(temperature=1e-60),
              dict(temperature=1e60), dict(k=-1), dict(k=129), dict(rows=1 << 60), dict(stride=1 << 62)]
    gradient = [dict(out_stride=vocab - 1), dict(out=p(out) + 2), dict(out=p(host)), dict(out=p(z) + 4),
                dict(out=p(z), out_stride=vocab + 1), dict(out_stride=1 << 62)]
    for name, good, wrong in (
            ("qn_logprobs", fwd, common + [
                dict(tokens=0), dict(tokens=p(t) + 4), dict(tokens=p(host)), dict(logprob=p(host)), dict(lse=p(host)),
                dict(entropy=p(f[2]) + 1), dict(top=0), dict(top_lp=0), dict(k=0), dict(logprob=p(z)),
                dict(top_lp=p(z) + 400), dict(top=p(z)),
                dict(logprob=0, lse=0, entropy=0, k=0, top=0, top_lp=0)]),
            ("qn_logprobs_backward", bwd, common + gradient + [
                dict(tokens=0), dict(vocab=qn.QN_GRAD_MAX_VOCAB + 1, stride=qn.QN_GRAD_MAX_VOCAB + 1),
                dict(dlp=0, dlse=0, dh=0, k=0, dtop=0), dict(top=0), dict(dtop=0), dict(k=0), dict(out=0), dict(dlp=p(host)), dict(top=p(top) + 4)]),
            ("qn_distill", dis, common + gradient + [
                dict(k=0), dict(token=0), dict(value=0), dict(loss=0), dict(value_dtype=2), dict(teacher=2),
                dict(teacher=-1), dict(weight=p(host)), dict(loss=p(z)), dict(vocab=qn.QN_GRAD_MAX_VOCAB + 1,
                                                                              stride=qn.QN_GRAD_MAX_VOCAB + 1)])):
        for change in wrong:
            assert call(name, good, **change) == bad, (name, change)
        assert call(name, good) == qn.QN_OK, name
    torch.cuda.synchronize()

    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_logprobs(z.cpu(), t, f[0])
    with pytest.raises(TypeError):
        qn.qn_logprobs(z.half(), t, f[0])
    with pytest.raises(ValueError, match="tokens"):
        qn.qn_logprobs(z, t.int(), f[0])
    with pytest.raises(ValueError, match="logprob"):
        qn.qn_logprobs(z, t, f[0][:2])
    with pytest.raises(ValueError, match="contiguous rows"):
        qn.qn_logprobs(z.t(), t, f[0])
    with pytest.raises(ValueError, match="contiguous rows"):
        qn.qn_logprobs(z[:1].expand(4, vocab), t, f[0])
    with pytest.raises(ValueError, match="go together"):
        qn.qn_logprobs(z, top_token=top)
    with pytest.raises(ValueError, match="dlogits"):
        qn.qn_logprobs_backward(z, out[:, :50], tokens=t, d_logprob=f[0])
    with pytest.raises(ValueError, match="teacher_value"):
        qn.qn_distill(z, top, top_lp[:, :2], f[0])
    with pytest.raises(qn.QNError):
        qn.qn_logprobs(z, t)  # no output
    with pytest.raises(qn.QNError):
        qn.qn_distill(z, top, top_lp, f[0], temperature=-2.0)
