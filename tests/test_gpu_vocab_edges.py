"""The operators over a vocabulary where a row, a size or an argument is out of the ordinary.

Tolerances are those of test_gpu_vocab.py, which derives them: 5e-6 (1 + |value|) for numbers per row, 1e-5 of the summed
magnitudes of its terms for an element of a gradient, and 2^-8 of it on top where it is stored as bf16.
"""
import math

import pytest
import torch

import vocab_reference as ref
from test_gpu_vocab import (DTYPES, check_backward, check_distill, check_logprobs, close, make_teacher,
                            some_tokens, upstream)

pytestmark = pytest.mark.gpu

INF = math.inf


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import qn as mod

    assert torch.cuda.is_available()
    mod.lib()
    return mod


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(700, 2048), (1300, 5003), (400, 40001), (2, 40001), (1, 262144)])
def test_alternatives_among_more_ties_than_are_collected(qn, rows, vocab, dtype):
    """More than 1024 equal logits at the top of most rows, and ordinary rows between them: the choice between the quick
    and the exhaustive selection has to be the same in every thread, row by row and launch by launch."""
    z = ref.make_logits(rows, vocab, dtype, rows)
    z[::3] = 4.0
    z[1::3, vocab // 4:] = 60.0
    tokens = some_tokens(rows, vocab, 6)
    for k in (5, 128):
        _, lse, _, top, _ = check_logprobs(qn, z, tokens, k)
        for _ in range(20):
            again, again_lse = torch.zeros_like(top), torch.zeros_like(lse)
            qn.qn_logprobs(z, lse=again_lse, top_token=again, top_logprob=torch.empty((rows, k), device="cuda"))
            assert torch.equal(again, top) and torch.equal(again_lse, lse)


@pytest.mark.parametrize("dtype", DTYPES)
def test_largest_vocabulary_of_the_forward_call(qn, dtype):
    """2^31 - 65 logits, the few that are not masked near the end, in a form that only the exhaustive paths take."""
    vocab = (1 << 31) - 65
    low = torch.finfo(dtype).min
    z = torch.full((1, vocab), -INF, dtype=dtype, device="cuda")
    z[0, -1] = low
    tokens = torch.tensor([vocab - 1], device="cuda")
    lp, lse, ent = (torch.zeros(1, device="cuda") for _ in range(3))
    top, top_lp = torch.zeros((1, 3), dtype=torch.int64, device="cuda"), torch.zeros((1, 3), device="cuda")

    def numbers():
        qn.qn_logprobs(z, tokens, lp, lse=lse, entropy=ent, top_token=top, top_logprob=top_lp)
        return float(lp), float(lse), float(ent), top[0].tolist(), top_lp[0].tolist()

    assert numbers() == (0.0, float(torch.tensor(low, dtype=dtype).float()), 0.0, [vocab - 1, -1, -1], [0.0, -INF, -INF])
    z[0, -2] = low
    z[0, 5] = low
    a, b, c, d, e = numbers()
    assert d == [5, vocab - 2, vocab - 1] and all(abs(x + math.log(3)) < 1e-5 for x in e + [a]) and abs(c - math.log(3)) < 1e-5
    z[0, vocab - 300] = 2.0
    assert numbers()[3] == [vocab - 300, 5, vocab - 2] and float(lse) == 2.0 and float(lp) < -3e38


# ---- distillation: a list far above or below the rest of the vocabulary ---------------------------------------------

# the first four sizes go to the kernel for small problems, the others (rows beyond 256 KB) to the pipeline
GAP_SHAPES = [(5, 40), (5, 1000), (300, 5003), (4, 40001), (4, 140001), (3, 300001)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", GAP_SHAPES)
@pytest.mark.parametrize("gap,temperature", [(80.0, 1.0), (100.0, 1.0), (300.0, 1.0), (30.0, 0.1), (600.0, 1.5)])
def test_distill_list_far_above_or_below_the_rest(qn, rows, vocab, gap, temperature, dtype):
    """What is left to the rest of the vocabulary, or to the list, is far below the smallest float: neither the loss nor
    the gradient may lose it."""
    k = 4
    z = ref.make_logits(rows, vocab, dtype, vocab)
    token = ref.make_logits(rows, vocab, torch.float32, 3).topk(k, 1).indices
    value = torch.tensor([-0.1, -4.0, -5.0, -5.0], device="cuda").expand(rows, k).contiguous()
    on = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda").scatter_(1, token, True)
    above = on.clone()
    above[1::4] = False
    above[1::4].scatter_(1, token[1::4, 2:3], True)  # one of the list alone
    above[2::4] = ~on[2::4]  # the rest
    above[3::4] = ~on[3::4] & (torch.arange(vocab, device="cuda") % 16 == 5)  # some of the rest
    z = torch.where(above, z.float() + gap, z.float()).to(dtype)
    weight = torch.rand(rows, device="cuda") + 0.5
    for logprobs in (True, False):
        loss, out = check_distill(qn, z, token, value, logprobs, temperature, weight)
        assert bool(torch.isfinite(loss).all()) and bool(torch.isfinite(out).all())


@pytest.mark.parametrize("vocab", [1000, 140001])
def test_distill_one_listed_token_leads(qn, vocab):
    """One listed logit of 100 above zeros, ln q = -0.1: by hand, p_r = (vocab - 1) e^-100 and every other gradient is
    -q_r / (vocab - 1)."""
    z = torch.zeros((1, vocab), device="cuda")
    z[0, 7] = 100.0
    token, value = torch.full((1, 1), 7, device="cuda"), torch.full((1, 1), -0.1, device="cuda")
    loss, out = check_distill(qn, z, token, value, True)
    q = math.exp(float(value))
    want = q * math.log(q) + (1 - q) * (math.log(1 - q) + 100 - math.log(vocab - 1))
    assert abs(float(loss) - want) < 5e-5
    assert abs(float(out[0, 3]) * (vocab - 1) + 1 - q) < 1e-6 and abs(float(out.double().sum())) < 1e-6


# ---- distillation: teacher and student masked alike -------------------------------------------------------------------


def distill_list_alone64(z, token, value, temperature):
    """Loss, gradient and sizes of their terms for a student that masks all but listed tokens, q_r = 0."""
    here = token >= 0
    logp = torch.log_softmax(z.double() / temperature, 1)
    v = torch.where(here, value.double(), -INF)
    q = v.exp()
    at = token.clamp(min=0)
    terms = torch.where(q > 0, q * (v - logp.gather(1, at)), 0.0)
    q_all = torch.zeros_like(logp).scatter_add_(1, at, q)
    p, mass = logp.exp(), q.sum(1, keepdim=True)
    return terms.sum(1), (mass * p - q_all) / temperature, (mass * p + q_all) / temperature


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(2000, 512), (600, 9001), (7, 140001), (3, 300001)])
@pytest.mark.parametrize("temperature", [1.0, 2.0])
def test_distill_teacher_and_student_masked_alike(qn, rows, vocab, temperature, dtype):
    """Fewer allowed tokens than alternatives: the list names all of them, and 1 - sum q is what rounding left of it."""
    k, allowed = 20, 10
    z = ref.make_logits(rows, vocab, dtype, 12)
    keep = ref.make_logits(rows, vocab, torch.float32, 13).topk(allowed, 1).indices
    z = torch.full_like(z, -INF).scatter_(1, keep, z.gather(1, keep))
    top, top_lp = torch.empty((rows, k), dtype=torch.int64, device="cuda"), torch.empty((rows, k), device="cuda")
    qn.qn_logprobs(z, top_token=top, top_logprob=top_lp, temperature=temperature)
    assert bool((top[:, :allowed] >= 0).all()) and bool((top[:, allowed:] == -1).all())
    for value in (top_lp, top_lp.bfloat16()):
        loss, out, again = torch.empty(rows, device="cuda"), torch.empty_like(z), torch.empty(rows, device="cuda")
        qn.qn_distill(z, top, value, loss, dlogits=out, temperature=temperature)
        qn.qn_distill(z, top, value, again, temperature=temperature)
        want, grad, size = distill_list_alone64(z, top, value, temperature)
        close(loss, want, torch.full_like(want, 5e-6 * 20), "loss")
        assert torch.equal(loss, again)
        bound = 1e-5 * size + 1e-30 + (2.0 ** -8 * grad.abs() + 2.0 ** -133 if dtype == torch.bfloat16 else 0.0)
        close(out, grad, bound, "dlogits")
        if value is top_lp:
            assert float(loss.abs().max()) < 1e-5 and float(out.float().abs().max()) < 1e-5


def test_distill_what_the_student_masks_and_the_teacher_does_not_is_infinite(qn):
    """More left for the rest than rounding leaves: the loss stays +inf."""
    for value_dtype, left in ((torch.float32, 1e-3), (torch.bfloat16, 0.2)):
        for vocab in (600, 300001):
            z = torch.full((3, vocab), -INF, device="cuda")
            z[:, 5:9] = 1.0
            token = torch.tensor([[5, 6, 7, 8, -1]], device="cuda").expand(3, 5).contiguous()
            value = torch.full((3, 5), math.log((1 - left) / 4), device="cuda").to(value_dtype)
            loss, out = torch.empty(3, device="cuda"), torch.empty_like(z)
            qn.qn_distill(z, token, value, loss, dlogits=out)
            assert bool((loss == INF).all()) and bool(torch.isfinite(out).all())


# ---- backward: the size of the upstream gradients ----------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(6, 50), (6, 9001), (3, 150001)])
def test_backward_of_large_upstream_gradients_and_masked_tokens(qn, rows, vocab, dtype):
    """A scaled loss: a masked token's gradient is its sparse terms alone, however large the entropy's factor is."""
    z = ref.make_logits(rows, vocab, dtype, 4)
    z[:, ::3] = -INF
    t = torch.full((rows,), 7, device="cuda")
    top = torch.tensor([3, 4], device="cuda").expand(rows, 2).contiguous()  # token 3 is masked
    for size in (1e6, 1e10, 1e15):
        out = check_backward(qn, z, t, 1.0, size * upstream(rows, 1), None, size * upstream(rows, 2), top,
                             size * upstream(rows, 3, 2))
        assert bool(torch.isfinite(out).all())


# ---- tokens that are not in the vocabulary -------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [60, 9001, 150001])
def test_gradients_of_a_token_that_is_not_in_the_vocabulary(qn, vocab, dtype):
    """NaN in its whole row, also where every token is masked; its neighbours keep theirs."""
    z = ref.make_logits(4, vocab, dtype, 9)
    z[1] = -INF
    z[2] = -INF
    t = torch.tensor([3, vocab, 3, vocab + 5], device="cuda")
    g = torch.ones(4, device="cuda")
    out, loss = torch.zeros_like(z), torch.zeros(4, device="cuda")
    for entropy in (None, g):
        out.zero_()
        qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g, d_entropy=entropy)
        assert out.isnan().all(1).tolist() == [False, True, False, True] and bool(torch.isfinite(out[::2]).all())
    qn.qn_logprobs_backward(z, out, top_token=t[:, None].contiguous(), d_top_logprob=g[:, None].contiguous())
    assert out.isnan().all(1).tolist() == [False, True, False, True]
    for teacher in (qn.QN_TEACHER_LOGITS, qn.QN_TEACHER_LOGPROBS):
        out.zero_()
        qn.qn_distill(z, torch.stack([t, t * 0 + 1], 1), torch.full((4, 2), -1.0, device="cuda"), loss, dlogits=out,
                      teacher=teacher)
        assert out.isnan().all(1).tolist() == [False, True, False, True] and bool(torch.isfinite(out[::2]).all())
        assert loss.isnan().tolist() == [False, True, False, True] and loss[2] == INF


@pytest.mark.parametrize("vocab", [60, 150001])
def test_padding_may_name_any_token(qn, vocab):
    """Rows whose upstream gradients are all 0 are padding whatever they hold, tokens outside the vocabulary included."""
    z = ref.make_logits(3, vocab, torch.float32, 9)
    t = torch.tensor([3, vocab, vocab + 7], device="cuda")
    g = torch.tensor([1.0, 0.0, 0.0], device="cuda")
    out = torch.ones_like(z)
    qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g, d_entropy=g, top_token=t[:, None].contiguous(),
                            d_top_logprob=g[:, None].contiguous())
    assert bool((out[1:] == 0).all()) and bool(torch.isfinite(out[0]).all()) and float(out[0].abs().max()) > 0


# ---- arguments -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(5, 33), (3, 8192), (4, 150001), (3, 160000)])
def test_gradient_interleaved_with_the_logits(qn, rows, vocab, dtype):
    """Logits and gradient as the two halves of one buffer's rows, whichever comes first."""
    near = ref.make_logits(rows, vocab, dtype, 2)
    t, g = some_tokens(rows, vocab, 1), upstream(rows, 1)
    token, value = make_teacher(near, 5, 1.0, True, 1)
    loss, want_loss = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    for swap in (0, 1):
        store = torch.zeros((rows, 2 * vocab), dtype=dtype, device="cuda")
        halves = (store[:, :vocab], store[:, vocab:])
        z, out = halves[swap], halves[1 - swap]
        z.copy_(near)
        qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g, d_entropy=g)
        apart = torch.zeros((rows, 2 * vocab), dtype=dtype, device="cuda")[:, :vocab]
        qn.qn_logprobs_backward(z, apart, tokens=t, d_logprob=g, d_entropy=g)
        assert torch.equal(out, apart) and torch.equal(z, near)
        qn.qn_distill(z, token, value, loss, dlogits=out)
        qn.qn_distill(z, token, value, want_loss, dlogits=apart)
        assert torch.equal(out, apart) and torch.equal(z, near) and torch.equal(loss, want_loss)


def test_gradient_that_shares_elements_with_the_logits_is_refused(qn):
    rows, vocab = 3, 10
    store = torch.zeros(200, device="cuda")
    t, g, loss = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.ones(rows, device="cuda"), torch.zeros(rows, device="cuda")
    z = store.as_strided((rows, vocab), (25, 1), 30)
    token, value = torch.zeros((rows, 1), dtype=torch.int64, device="cuda"), torch.zeros((rows, 1), device="cuda")

    def calls(out):
        yield lambda: qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g)
        yield lambda: qn.qn_distill(z, token, value, loss, dlogits=out)

    for stride, offset in ((25, 21), (25, 39), (25, 46), (25, 14), (24, 40), (30, 0)):
        for call in calls(store.as_strided((rows, vocab), (stride, 1), offset)):
            with pytest.raises(qn.QNError):
                call()
    for stride, offset in ((25, 20), (25, 40), (25, 45), (25, 15), (25, 110), (10, 0)):
        for call in calls(store.as_strided((rows, vocab), (stride, 1), offset)):
            call()


def test_temperatures_whose_inverse_does_not_fit_are_refused(qn):
    """1 / T still fits in 32 bits for these, log2(e) / T does not; the smallest that fit give numbers."""
    z = ref.make_logits(2, 50, torch.float32, 1)
    z[:, 7] = 100.0
    t, v = torch.full((2,), 7, device="cuda"), torch.zeros(2, device="cuda")
    token, value = t[:, None].contiguous(), torch.zeros((2, 1), device="cuda")
    out = torch.zeros_like(z)
    for temperature in (3e-39, 4e-39):
        for call in (lambda x: qn.qn_logprobs(z, t, v, temperature=x),
                     lambda x: qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=v, temperature=x),
                     lambda x: qn.qn_distill(z, token, value, v, dlogits=out, temperature=x)):
            with pytest.raises(qn.QNError):
                call(temperature)
    qn.qn_logprobs(z, t, v, temperature=5e-39)
    assert v.tolist() == [0.0, 0.0]


def test_no_alternatives_of_width_zero(qn):
    """top_token [rows][0] is k = 0, as d_top_logprob [rows][0] is."""
    z = ref.make_logits(4, 100, torch.float32, 1)
    t, g = some_tokens(4, 100, 1), upstream(4, 1)
    none, none_lp = torch.empty((4, 0), dtype=torch.int64, device="cuda"), torch.empty((4, 0), device="cuda")
    lp, want = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    qn.qn_logprobs(z, t, want)
    qn.qn_logprobs(z, t, lp, top_token=none, top_logprob=none_lp)
    assert torch.equal(lp, want)
    out, same = torch.zeros_like(z), torch.zeros_like(z)
    qn.qn_logprobs_backward(z, out, tokens=t, d_logprob=g)
    qn.qn_logprobs_backward(z, same, tokens=t, d_logprob=g, top_token=none, d_top_logprob=none_lp)
    assert torch.equal(out, same)
    with pytest.raises(ValueError, match="top_logprob"):
        qn.qn_logprobs(z, t, lp, top_token=none, top_logprob=torch.empty((4, 1), device="cuda"))


# ---- backward: rows whose maximum is far above what comes before it --------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(6, 1000), (5, 30000), (300, 140001), (4, 150000), (40, 300001)])
@pytest.mark.parametrize("temperature,step", [(1.0, 60.0), (1.0, 200.0), (0.05, 3.0)])
def test_backward_of_the_entropy_where_the_maximum_rises_in_steps(qn, rows, vocab, temperature, step, dtype):
    """Each tenth of a row is a step above the one before it (and the other way round in every other row): what was
    summed before a step weighs nothing after it."""
    z = ref.make_logits(rows, vocab, dtype, vocab)
    rise = step * torch.div(10 * torch.arange(vocab, device="cuda"), vocab, rounding_mode="floor")
    z = (z.float() + torch.where(torch.arange(rows, device="cuda")[:, None] % 2 == 0, rise, rise.flip(0))).to(dtype)
    t = torch.full((rows,), vocab - 1, device="cuda")
    check_backward(qn, z, t, temperature, None, None, upstream(rows, 1), None, None)
    check_backward(qn, z, t, temperature, upstream(rows, 2), upstream(rows, 3), upstream(rows, 4), None, None)
    check_logprobs(qn, z, t, 3, temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("fill", ["lowest", -10000.0])
@pytest.mark.parametrize("rows,vocab", [(500, 600), (40, 9001), (7, 140001), (3, 300001)])
def test_distill_teacher_and_student_masked_alike_by_a_very_low_number(qn, rows, vocab, fill, dtype):
    """The same where the mask is the type's lowest value, or -10000: all allowed tokens are listed, some of the others too, and the
    student gives the rest e^-9000 or less."""
    k, allowed = 20, 10
    z = ref.make_logits(rows, vocab, dtype, 12)
    keep = ref.make_logits(rows, vocab, torch.float32, 13).topk(allowed, 1).indices
    z = torch.full_like(z, torch.finfo(dtype).min if fill == "lowest" else fill).scatter_(1, keep, z.gather(1, keep))
    top, top_lp = torch.empty((rows, k), dtype=torch.int64, device="cuda"), torch.empty((rows, k), device="cuda")
    qn.qn_logprobs(z, top_token=top, top_logprob=top_lp)
    assert bool((top >= 0).all())
    for value in (top_lp, top_lp.bfloat16()):
        loss, out, again = torch.empty(rows, device="cuda"), torch.empty_like(z), torch.empty(rows, device="cuda")
        qn.qn_distill(z, top, value, loss, dlogits=out)
        qn.qn_distill(z, top, value, again)
        want, grad, size = distill_list_alone64(z, top, value, 1.0)
        close(loss, want, torch.full_like(want, 5e-6 * 20), "loss")
        assert torch.equal(loss, again)
        bound = 1e-5 * size + 1e-30 + (2.0 ** -8 * grad.abs() + 2.0 ** -133 if dtype == torch.bfloat16 else 0.0)
        close(out, grad, bound, "dlogits")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("vocab", [300, 150001])
def test_distill_of_a_masked_token_that_the_teacher_weighs_less_than_the_smallest_float(qn, vocab, logprobs, dtype):
    """q = e^-200 is 0 in 32 bits and the student masks it: +inf all the same; not so where the teacher masks it too, with
    -inf or the lowest value."""
    z = ref.make_logits(4, vocab, dtype, 3)
    token = torch.tensor([3, 8, 9], device="cuda").expand(4, 3).contiguous()
    z[:3, 8] = -INF
    value = torch.tensor([-0.5, -200.0, -2.0], device="cuda").repeat(4, 1)
    value[1, 1], value[2, 1] = -INF, torch.finfo(torch.float32).min
    loss, out = check_distill(qn, z, token, value, logprobs)
    assert loss[0] == INF and bool(torch.isfinite(loss[1:]).all()) and bool(torch.isfinite(out).all())


# ---- many small terms beside a large one -----------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(400, 30000), (700, 131072), (300, 262144), (2, 393000)])
def test_small_terms_beside_the_peak_are_not_lost(qn, rows, vocab, dtype):
    """One token at 0 and all others near -16: each of them is below half of the last bit of the peak's term, together they
    are a few per cent of the sum."""
    z = (ref.make_logits(rows, vocab, torch.float32, 2, spread=0.05) - 16.5).to(dtype)
    at = torch.arange(rows, device="cuda") * 7 % 64
    z[torch.arange(rows, device="cuda"), at] = 0.0
    check_logprobs(qn, z, at, 3)
    g = upstream(rows, 1)
    check_backward(qn, z, at + 100, 1.0, g, None, g, None, None)
    token, value = make_teacher(z, 2, 1.0, True, 1)
    token[:, 0] = at + 500  # the peak is off the list
    check_distill(qn, z, token, value, True)
