"""qn_policy and qn_preference against their 64-bit forms.

Tolerances.  qn_policy: a log probability and an entropy are good to 5e-6 (1 + |value|) (test_gpu_vocab.py derives it); what that is in
the loss and in the slope comes from objective_reference (``per``: for an error of 1), and 1e-6 of the terms' sizes for the
arithmetic after it; a gradient's element has 1e-5 of its terms' sizes, and 2^-8 of it where it is stored as bf16.
qn_preference: sums in 64 bits of products of numbers in 32 (exact), rounded once: 2^-23 of each result and 1e-13 of what is
added up, times the slope's own slope, which is at most 1 / 4 (logistic) or 2 / beta^2 (squared).
"""
import math

import pytest
import torch

import objective_reference as ref
import vocab_reference

pytestmark = pytest.mark.gpu

INF = math.inf
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import qn as mod

    assert torch.cuda.is_available()
    mod.lib()
    return mod


# ---- policy --------------------------------------------------------------------------------------------------------------


def policy_inputs(z, temperature, seed, low=0.2, high=0.2, dual=0.0):
    """Tokens, the older policy's and the reference's log probabilities, advantages; no ratio within 1e-3 of a bound."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab = z.shape
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    logp = torch.log_softmax(z.double() / temperature, 1).gather(1, tokens[:, None])[:, 0]
    logp = torch.where(torch.isfinite(logp), logp, -5.0)
    change = 0.3 * torch.randn(rows, generator=gen, device="cuda", dtype=torch.float64)
    for bound in (1 - low, 1 + high, dual):
        if 0 < bound < INF:
            change = torch.where((change - math.log(bound)).abs() < 1e-3, change + 3e-3, change)
    return (tokens, (logp - change).float(), (logp + 0.5 * torch.randn(rows, generator=gen, device="cuda")).float(),
            torch.randn(rows, generator=gen, device="cuda"))


def check_policy(qn, z, tokens, old, reference, advantage, weight=None, temperature=1.0, low=0.2, high=0.2, dual=0.0, kl=0.0,
                 bonus=0.0, out=None, entropy=True, stream=None):
    rows = z.shape[0]
    before = z.clone()
    loss, lp, ent = (torch.full((rows,), 9.0, device="cuda") for _ in range(3))
    grad = torch.full_like(z, 9.0) if out is None else out
    args = dict(ref_logprob=reference if kl else None, weight=weight, clip_low=low, clip_high=high, dual=dual, kl=kl, entropy_bonus=bonus,
                temperature=temperature, stream=stream)
    torch.cuda.synchronize()  # `stream` waits for no other, and no other for it
    qn.qn_policy(z, tokens, old, advantage, loss, dlogits=grad, logprob=lp, entropy=ent if entropy else None, **args)
    torch.cuda.synchronize()
    want_loss, want_lp, want_ent, want, per, size, per_grad, ratio = ref.policy64(before, tokens, old, reference, advantage, weight,
                                                                               temperature, low, high, dual, kl, bonus)
    for bound in (1 - low, 1 + high, dual):  # the inputs are such that rounding cannot move a ratio over a bound
        assert not bool((((ratio - bound).abs() < 1e-4) & (bound > 0)).any())
    off = 5e-6 * (1 + torch.where(torch.isfinite(want_lp), want_lp.abs(), 0.0))
    off_h = 5e-6 * (1 + torch.nan_to_num(want_ent).abs())

    def close(got, value, bound):
        same = (got.double() == value) | (torch.isnan(got) & torch.isnan(value))
        assert bool((same | ((got.double() - value).abs() <= bound)).all()), float(
            torch.where(same, 0.0, (got.double() - value).abs() / (bound + 1e-300)).nan_to_num(1e300).max())

    close(lp, want_lp, off)
    if entropy:
        close(ent, want_ent, off_h)
    base = 1e-6 * (torch.nan_to_num(want_loss, posinf=0.0).abs() + per.nan_to_num() + abs(bonus) * torch.nan_to_num(want_ent).abs() + kl)
    close(loss, want_loss, torch.nan_to_num(per, posinf=0.0) * off + abs(bonus) * off_h + base)
    bound = torch.nan_to_num(per_grad, posinf=0.0) * off[:, None] + 1e-5 * torch.nan_to_num(size, posinf=0.0)
    if z.dtype == BF16:
        bound = bound + 2.0 ** -8 * torch.nan_to_num(want).abs() + 1e-40
    close(grad, want, bound)
    # the loss alone gives the same numbers
    alone = torch.full((rows,), 9.0, device="cuda")
    if out is None:
        torch.cuda.synchronize()
        qn.qn_policy(z, tokens, old, advantage, alone, logprob=lp, **args)
        torch.cuda.synchronize()
        same = (alone == loss) | (torch.isnan(alone) & torch.isnan(loss))
        assert bool((same | ((alone - loss).abs() <= 2e-6 * (1 + loss.abs()) + 2 * (torch.nan_to_num(per, posinf=0.0) * off).float())).all())
        assert torch.equal(z, before) or bool(torch.isnan(z).any())
    return loss, grad


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab,pad,offset", [(1, 1, 0, 0), (1, 2, 1, 1), (3, 29, 3, 1), (7, 1000, 0, 0), (130, 4099, 5, 2),
                                                   (33, 32000, 0, 0), (3, 131072, 8, 0), (2, 262143, 1, 3), (1, 393208, 0, 0),
                                                   (900, 50001, 0, 0), (400, 131072, 0, 0)])
@pytest.mark.parametrize("kl,bonus,dual", [(0.0, 0.0, 0.0), (0.1, 0.02, 3.0)])
def test_policy_over_sizes_and_places(qn, dtype, rows, vocab, pad, offset, kl, bonus, dual):
    z = vocab_reference.make_logits(rows, vocab, dtype, rows + vocab, pad, offset)
    tokens, old, reference, advantage = policy_inputs(z, 1.3, rows, dual=dual)
    weight = torch.rand(rows, device="cuda") + 0.5
    weight[2::5] = 0.0
    tokens[4::7] = -1
    check_policy(qn, z, tokens, old, reference, advantage, weight, 1.3, dual=dual, kl=kl, bonus=bonus, entropy=bonus != 0)


@pytest.mark.parametrize("low,high,dual", [(0.0, 0.0, 0.0), (1.0, INF, 0.0), (0.1, 0.4, 2.0), (1.0, 0.3, 1.5)])
def test_policy_bounds(qn, low, high, dual):
    """Both signs of the advantage and 0, ratios on every side of every bound."""
    z = vocab_reference.make_logits(300, 777, F32, 5)
    tokens, old, reference, advantage = policy_inputs(z, 1.0, 3, low, high, dual)
    advantage[::6] = 0.0
    old[1::4] -= 1.0  # ratios of e
    old[2::4] += 1.0
    check_policy(qn, z, tokens, old, reference, advantage, None, 1.0, low, high, dual, kl=0.3, bonus=-0.1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(40, 500), (1500, 40001)])
def test_policy_of_rows_out_of_the_ordinary(qn, dtype, rows, vocab):
    """Masked tokens, masked vocabularies, empty rows, NaN and infinities in rows, padding and side inputs."""
    z = vocab_reference.make_logits(rows, vocab, dtype, 8)
    tokens, old, reference, advantage = policy_inputs(z, 1.0, 4)
    weight = torch.ones(rows, device="cuda")
    each = torch.arange(rows, device="cuda")
    z[each[1::16], tokens[1::16]] = -INF           # the token is masked
    z[each[2::16], tokens[2::16]] = -INF           # by the reference too
    reference[2::16] = -INF
    z[3::16] = -INF                                # empty
    z[4::16] = -INF
    z[each[4::16], tokens[4::16]] = 1.0            # nothing but the token
    z[5::16, 0] = INF
    z[6::16, vocab // 2] = math.nan
    z[7::16] = math.nan                            # padding, whatever it holds
    weight[7::16] = 0.0
    z[8::16] = INF
    tokens[8::16] = -3
    tokens[9::16] = vocab                          # not in the vocabulary
    old[10::16] = math.nan
    advantage[11::16] = math.nan
    reference[12::16] = math.nan
    z[13::16] = torch.finfo(dtype).min             # uniform
    old[13::16] = -math.log(vocab) - 0.05
    reference[13::16] = -math.log(vocab)
    reference[14::16] = -INF                       # the reference masks what the policy took
    z[15::16, 1:] = -INF                           # all but one
    tokens[15::16] = 0
    for kl, bonus in ((0.0, 0.0), (0.2, 0.05)):
        check_policy(qn, z, tokens, old, reference, advantage, weight, kl=kl, bonus=bonus, entropy=bonus != 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,vocab", [(5, 1000), (700, 60000)])
def test_policy_gradient_in_place_and_elsewhere(qn, dtype, rows, vocab):
    z = vocab_reference.make_logits(rows, vocab, dtype, 2)
    args = policy_inputs(z, 1.0, 9)
    want = check_policy(qn, z, *args, kl=0.1, bonus=0.01)[1]
    for place in ("odd", "between", "stream", "in place"):
        if place == "odd":
            out = torch.full((rows * (vocab + 3) + 1,), 9.0, dtype=dtype, device="cuda").as_strided((rows, vocab), (vocab + 3, 1), 1)
            same = check_policy(qn, z, *args, kl=0.1, bonus=0.01, out=out)[1]
            assert torch.allclose(same.float(), want.float(), rtol=2 ** -7, atol=1e-7)
        elif place == "between":
            store = torch.empty((rows, 2 * vocab), dtype=dtype, device="cuda")
            store[:, :vocab] = z
            check_policy(qn, store[:, :vocab], *args, kl=0.1, bonus=0.01, out=store[:, vocab:])
        elif place == "stream":
            stream = torch.cuda.Stream()
            torch.cuda.synchronize()
            check_policy(qn, z, *args, kl=0.1, bonus=0.01, stream=stream)
        else:
            mine = z.clone()
            loss, got = check_policy(qn, mine, *args, kl=0.1, bonus=0.01, out=mine)
            assert torch.equal(got, want)


def test_policy_gradient_is_the_difference_of_its_losses(qn):
    """(L(z + h e) - L(z - h e)) / 2 h in fp32: the loss is good to a few 1e-7, so with h = 0.05 a difference to 1e-5, beside the
    third-order term h^2 / 6 times a third derivative of order 1, 5e-4."""
    z = vocab_reference.make_logits(6, 50, F32, 3)
    tokens, old, reference, advantage = policy_inputs(z, 1.0, 6)
    args = dict(ref_logprob=reference, kl=0.3, entropy_bonus=0.1, clip_low=1.0, clip_high=INF)
    loss, grad = torch.empty(6, device="cuda"), torch.empty_like(z)
    qn.qn_policy(z, tokens, old, advantage, loss, dlogits=grad, **args)
    for i in (0, 17, 49, *tokens.tolist()):
        both = []
        for h in (0.05, -0.05):
            moved = z.clone()
            moved[:, i] += h
            qn.qn_policy(moved, tokens, old, advantage, loss, **args)
            both.append(loss.clone())
        assert torch.allclose((both[0] - both[1]) / 0.1, grad[:, i], atol=3e-3)


def test_policy_captured_and_replayed(qn):
    z = vocab_reference.make_logits(64, 5000, BF16, 3)
    tokens, old, reference, advantage = policy_inputs(z, 1.0, 6)
    loss, grad = torch.empty(64, device="cuda"), torch.empty_like(z)
    qn.qn_policy(z, tokens, old, advantage, loss, dlogits=grad)
    want = loss.clone(), grad.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qn.qn_policy(z, tokens, old, advantage, loss, dlogits=grad)
    for _ in range(2):
        loss.zero_(), grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])


# ---- preference ------------------------------------------------------------------------------------------------------------


def preference_inputs(lengths, ref_dtype, seed, lead=0, behind=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    offsets = torch.tensor([lead] + [lead + sum(lengths[: i + 1]) for i in range(len(lengths))], device="cuda")
    tokens = int(offsets[-1]) + behind
    l = -torch.empty(tokens, device="cuda").exponential_(generator=gen)  # noqa: E741
    reference = None if ref_dtype is None else (l + 0.2 * torch.randn(tokens, generator=gen, device="cuda")).to(ref_dtype)
    weight = (torch.rand(tokens, generator=gen, device="cuda") < 0.7).float() * (1 + torch.arange(tokens, device="cuda") % 3)
    return l, offsets, reference, weight, torch.rand(len(lengths) // 2, generator=gen, device="cuda") + 0.5


def check_preference(qn, l, offsets, reference, weight, pair_weight, kind=0, beta=0.1, margin=0.0, smoothing=0.0, normalise=False,
                     split=False, stream=None):
    tokens, pairs = l.numel(), (offsets.numel() - 1) // 2
    loss, reward = torch.full((pairs,), 9.0, device="cuda"), torch.full((2 * pairs,), 9.0, device="cuda")
    grad = torch.full((tokens,), 7.0, device="cuda")
    args = dict(ref_logprob=reference, weight=weight, pair_weight=pair_weight, kind=kind, beta=beta, margin=margin, smoothing=smoothing,
                normalise=normalise, split=split, stream=stream)
    torch.cuda.synchronize()  # `stream` waits for no other, and no other for it
    qn.qn_preference(l, offsets, loss, d_logprob=grad, reward=reward, **args)
    torch.cuda.synchronize()
    want_loss, want_reward, want, size = ref.preference64(l, offsets, reference, weight, pair_weight, kind, beta, margin, smoothing,
                                                          normalise, split)
    both = size.view(2, pairs).t() if split else size.view(pairs, 2)
    off_h = 1e-13 * torch.nan_to_num(both.sum(1), posinf=0.0)
    curve = 0.25 if kind == 0 else 0.0 if kind == 1 else 2 / beta ** 2

    def close(got, value, bound):
        same = (got.double() == value) | (torch.isnan(got) & torch.isnan(value))
        assert bool((same | ((got.double() - value).abs() <= bound + 2.0 ** -23 * value.abs())).all())

    close(reward, want_reward, 1e-13 * torch.nan_to_num(size, posinf=0.0))
    steep = 1.0 if kind != 2 else torch.nan_to_num(2 * want_loss.sqrt() / beta, posinf=0.0)
    close(loss, want_loss, steep * off_h + curve * off_h ** 2 + 1e-14)
    largest = float(torch.nan_to_num(weight, nan=0.0, posinf=0.0).abs().max()) if weight is not None and weight.numel() else 1.0
    heavy = float(pair_weight.abs().max()) if pair_weight is not None else 1.0
    each = beta * (1.0 if not normalise else 10.0)
    close(grad, want, curve * float(off_h.max()) * largest * heavy * each + 1e-14 * largest * heavy * each)
    alone = torch.full((pairs,), 9.0, device="cuda")
    torch.cuda.synchronize()
    qn.qn_preference(l, offsets, alone, **args)
    torch.cuda.synchronize()
    assert bool(((alone == loss) | (torch.isnan(alone) & torch.isnan(loss))).all())
    return loss, reward, grad


LENGTHS = {"one token": [1, 1], "nothing": [0, 0], "one empty": [0, 5, 3, 0], "short": [3, 9, 31, 32, 33, 64, 1, 7],
           "ragged": [700, 3, 1, 1025, 0, 4000, 513, 512], "long": [70001, 65], "longer": [3, 300_000, 200_003, 5]}


@pytest.mark.parametrize("lengths", LENGTHS)
@pytest.mark.parametrize("ref_dtype", [None, F32, BF16])
@pytest.mark.parametrize("kind,smoothing,normalise,split", [(0, 0.0, False, False), (0, 0.1, True, True), (1, 0.0, False, True),
                                                            (2, 0.0, True, False)])
def test_preference_over_lengths(qn, lengths, ref_dtype, kind, smoothing, normalise, split):
    args = preference_inputs(LENGTHS[lengths], ref_dtype, 3, lead=5, behind=9)
    grad = check_preference(qn, *args, kind, 0.3, 0.2, smoothing, normalise, split)[2]
    # tokens of no sequence are left as they were
    assert bool((grad[:5] == 7).all()) and bool((grad[-9:] == 7).all())


@pytest.mark.parametrize("pairs,length", [(5000, 3), (600, 200), (100, 3000), (3, 40000)])
def test_preference_of_many_pairs(qn, pairs, length):
    lengths = [(7 * i * i + 3) % (2 * length) for i in range(2 * pairs)]
    args = preference_inputs(lengths, F32, 8)
    check_preference(qn, *args, beta=0.05)
    check_preference(qn, args[0], args[1], args[2], None, None, beta=0.05, split=True)
    weight = args[4]
    weight[::3] = 0.0
    check_preference(qn, *args[:4], weight, normalise=True)


def test_preference_masks_and_extremes(qn):
    l, offsets, reference, weight, pair_weight = preference_inputs([40] * 20, F32, 5)
    for i in range(20):
        a = 40 * i
        weight[a] = 1.0
        if i == 0:  # what does not count may be anything
            l[a + 1:a + 4] = torch.tensor([math.nan, -INF, INF])
            weight[a + 1:a + 4] = 0.0
        if i == 2:
            reference[a + 1], weight[a + 1] = math.nan, 0.0
        if i == 4:  # masked by both
            l[a] = reference[a] = -INF
        if i == 6:  # by the policy: the loss of its pair is +inf, the slope -beta
            l[a] = -INF
        if i == 9:  # the rejected one by the policy: the loss is 0
            l[a] = -INF
        if i == 10:
            reference[a] = -INF
        if i == 13:
            l[a] = math.nan
        if i == 14:  # nothing counts
            weight[a:a + 40] = 0.0
        if i in (16, 17):  # both infinite
            l[a] = -INF
    pair_weight[9] = 0.0
    l[18 * 40] = math.nan
    weight[18 * 40] = 1.0
    for kind in (0, 1, 2):
        for normalise in (False, True):
            for smoothing in (0.0, 0.2):
                check_preference(qn, l, offsets, reference, weight, pair_weight, kind, 0.3, 0.1, smoothing, normalise)
    # rewards of a thousand: the logistic loss is h itself on one side and 0 on the other
    big = preference_inputs([50, 50, 50, 50], None, 5)
    l = big[0].clone()
    l[:50], l[50:100], l[100:150], l[150:] = -300.0, 0.0, 0.0, -300.0
    check_preference(qn, l, big[1], None, None, None, beta=1.0)


def test_preference_masks_in_long_sequences(qn):
    """Tokens that both sides mask, and what does not count, past the tiles whose weights are kept."""
    lengths = [400_000, 30, 300_001, 290_000]
    l, offsets, reference, weight, pair_weight = preference_inputs(lengths, BF16, 5, lead=3, behind=2)
    l[::1001] = -INF
    reference[::1001] = -INF
    l[500::999], weight[500::999] = math.nan, 0.0
    for normalise in (False, True):
        check_preference(qn, l, offsets, reference, weight, pair_weight, beta=0.001, normalise=normalise)


@pytest.mark.parametrize("ref_dtype", [None, F32, BF16])
@pytest.mark.parametrize("kind,smoothing,normalise,split", [(0, 0.1, False, True), (0, 0.0, True, False), (1, 0.0, True, False),
                                                            (2, 0.0, False, True)])
def test_preference_of_short_pairs_with_long_ones_between(qn, ref_dtype, kind, smoothing, normalise, split):
    """More pairs than the device has room for blocks, short ones on average: one of nothing, one of nothing that counts, padding,
    masked tokens, long sequences among them, and a pair out of place."""
    pairs = 2501
    lengths = [(11 * i * i + 5) % 90 for i in range(2 * pairs)]
    lengths[7], lengths[2 * pairs - 3], lengths[2000], lengths[2001] = 9001, 5000, 0, 0
    l, offsets, reference, weight, pair_weight = preference_inputs(lengths, ref_dtype, 12, lead=3, behind=4)
    pair_weight[5::17] = 0.0
    at = offsets.tolist()
    weight[at[900]:at[902]] = 0.0
    weight[at[7] + 17:at[8]:31] = 0.0
    l[at[7] + 17:at[8]:31] = math.nan
    if reference is not None:
        l[1000::1013] = reference[1000::1013] = -INF
    else:
        weight[1000::1013] = 0.0
    offsets[-1] += 5
    loss, _, grad = check_preference(qn, l, offsets, reference, weight, pair_weight, kind, 0.3, 0.1, smoothing, normalise, split)
    assert bool(torch.isnan(loss[-1])) and bool((grad[:3] == 7).all()) and int(torch.isnan(loss).sum()) == 1


def test_preference_offsets_that_are_wrong(qn):
    """Every way to leave [0, tokens] or to go backwards, with a good pair beside each; nothing outside is touched."""
    good = [(0, 4), (4, 9)]
    for bad in (-1, 100, 1 << 40, -(1 << 62), (1 << 62)):
        at = torch.tensor([0, 4, bad, 12, 20], device="cuda")
        l = torch.randn(20, device="cuda")
        loss, reward, grad = check_preference(qn, l, at, None, None, None, beta=0.5, split=False)
        assert bool(torch.isnan(loss).all())
    at = torch.tensor([0, 4, 9, 25, 21], device="cuda")
    l = torch.randn(21, device="cuda")
    loss, _, _ = check_preference(qn, l, at, None, None, None)
    assert bool(torch.isfinite(loss[0])) and bool(torch.isnan(loss[1]))
    del good


def test_preference_gradient_is_the_difference_of_its_losses(qn):
    """In steps of 2^-6 of one token, which fp32 holds exactly: the difference is off by 2^-23 of the loss over 2^-5, 4e-6, and by
    (beta / 64)^2 / 6 of the third derivative, 1e-5 at beta = 0.5."""
    l, offsets, reference, weight, pair_weight = preference_inputs([5, 8, 2, 1], F32, 4)
    loss, grad = torch.empty(2, device="cuda"), torch.empty(16, device="cuda")
    for kind in (0, 2):
        args = dict(ref_logprob=reference, weight=weight, beta=0.5, kind=kind, smoothing=0.1)
        qn.qn_preference(l, offsets, loss, d_logprob=grad, **args)
        for i in range(16):
            both = []
            for h in (2.0 ** -6, -(2.0 ** -6)):
                moved = l.clone()
                moved[i] += h
                qn.qn_preference(moved, offsets, loss, **args)
                both.append(loss.double().sum())
            assert abs(float(both[0] - both[1]) * 32 - float(grad[i])) < 1e-4 * (1 + float(loss.max()))


def test_preference_captured_and_on_another_stream(qn):
    args = preference_inputs([3000, 2000] * 30, BF16, 5)
    torch.cuda.synchronize()
    want = check_preference(qn, *args, stream=torch.cuda.Stream())
    loss, grad = torch.empty(30, device="cuda"), torch.empty_like(args[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        qn.qn_preference(args[0], args[1], loss, d_logprob=grad, ref_logprob=args[2], weight=args[3], pair_weight=args[4])
    for _ in range(2):
        loss.zero_(), grad.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[2])


# ---- together, as they are used ---------------------------------------------------------------------------------------------


def test_a_run_of_all_of_them(qn):
    """Logits -> log probabilities -> preference loss -> gradient of the logits -> gradient of the weights -> clipped step; and the
    same chain in 64 bits through torch's own derivative.  The gradient of W is good to 1e-5 of its largest element (as in
    the distillation loop's test) and the first AdamW step is the gradient's sign times lr where it is not small beside eps."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    vocab, dim, lengths = 301, 16, [20, 12, 7, 30]
    rows = sum(lengths)
    x, w = torch.randn(rows, dim, generator=gen, device="cuda"), 0.3 * torch.randn(vocab, dim, generator=gen, device="cuda")
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    offsets = torch.tensor([0, 20, 32, 39, 69], device="cuda")
    reference = torch.log_softmax((x @ w.t()).double(), 1).gather(1, tokens[:, None])[:, 0].float()
    w = w + 0.05 * torch.randn(vocab, dim, generator=gen, device="cuda")
    z = x @ w.t()
    lp, d_lp, loss = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(2, device="cuda")
    half = torch.full((2,), 0.5, device="cuda")
    qn.qn_logprobs(z, tokens, lp)
    qn.qn_preference(lp, offsets, loss, d_logprob=d_lp, ref_logprob=reference, pair_weight=half, beta=0.5)
    qn.qn_logprobs_backward(z, z, tokens=tokens, d_logprob=d_lp)
    grad = z.t() @ x

    w64 = w.double().requires_grad_()
    lp64 = torch.log_softmax(x.double() @ w64.t(), 1).gather(1, tokens[:, None])[:, 0] - reference.double()
    sums = torch.stack([lp64[offsets[i]:offsets[i + 1]].sum() for i in range(4)])
    value = -torch.nn.functional.logsigmoid(0.5 * (sums[0::2] - sums[1::2]))
    want, = torch.autograd.grad(value.mean(), w64)
    assert torch.allclose(loss.double(), value.detach(), rtol=1e-5, atol=1e-5)
    assert float((grad.double() - want).abs().max()) <= 1e-5 * float(want.abs().max())

    m, v = torch.zeros_like(w), torch.zeros_like(w)
    step, sumsq = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    before = w.clone()
    with qn.qn_adam_create([w], [grad], [m], [v]) as plan:
        qn.qn_adam_norm(plan, sumsq)
        qn.qn_adam_step(plan, step, lr=1e-2, eps=1e-12, sumsq=sumsq, max_norm=0.5 * float(want.norm()))
    assert abs(float(sumsq) ** 0.5 / float(want.norm()) - 1) < 1e-4
    sure = want.abs() > 1e-3 * want.abs().max()
    assert torch.allclose((w - before)[sure], -1e-2 * torch.sign(want[sure]).float(), atol=1e-6)


# ---- refusals ----------------------------------------------------------------------------------------------------------------


def test_refusals(qn):
    z, t = torch.zeros((4, 8), device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    a, b, c, loss = (torch.zeros(4, device="cuda") for _ in range(4))

    def refused(kind, **change):
        args = dict(logits=z, tokens=t, old_logprob=a, advantage=b, loss=loss)
        with pytest.raises(kind):
            qn.qn_policy(**{**args, **change})

    refused(ValueError, tokens=None)
    refused(ValueError, tokens=t.int())
    refused(ValueError, tokens=t[:3])
    refused(ValueError, old_logprob=a.cpu())
    refused(ValueError, advantage=b.double())
    refused(ValueError, weight=a[:2])
    refused(ValueError, dlogits=z[:, :4])
    refused(TypeError, logits=z.half())
    refused(ValueError, logits=z.t())
    for change in (dict(kl=0.1), dict(kl=-0.1, ref_logprob=c), dict(clip_low=-0.1), dict(clip_low=1.5), dict(clip_high=-0.1),
                   dict(clip_low=math.nan), dict(dual=0.5), dict(dual=INF), dict(entropy_bonus=INF), dict(temperature=0.0),
                   dict(logprob=loss), dict(logprob=a), dict(entropy=b), dict(loss=a), dict(loss=z[0, :4]),
                   dict(loss=torch.zeros(8, device="cuda")[::2])):
        refused((qn.QNError, ValueError), **change)
    big = torch.zeros((1, qn.QN_GRAD_MAX_VOCAB + 1), device="cuda")
    one = torch.zeros(1, device="cuda")
    with pytest.raises(qn.QNError):
        qn.qn_policy(big, t[:1], one, one.clone(), one.clone())
    qn.qn_policy(z[:0], t[:0], a[:0], b[:0], loss[:0])  # nothing to do

    l, at = torch.zeros(6, device="cuda"), torch.tensor([0, 1, 3, 4, 6], device="cuda")  # noqa: E741
    two, four, six = torch.zeros(2, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros(6, device="cuda")

    def pref(error, **change):
        with pytest.raises(error):
            qn.qn_preference(**{**dict(logprob=l, offsets=at, loss=two), **change})

    pref(ValueError, loss=two.cpu())
    pref(ValueError, logprob=l.double())
    pref(ValueError, offsets=at.int())
    pref(ValueError, offsets=at[:4])
    pref(ValueError, reward=two)
    pref(ValueError, d_logprob=four)
    pref(TypeError, ref_logprob=six.half())
    pref(ValueError, weight=six.bfloat16())
    for change in (dict(beta=0.0), dict(beta=math.nan), dict(margin=INF), dict(smoothing=1.5), dict(smoothing=-0.1), dict(kind=3),
                   dict(d_logprob=l), dict(reward=l[:4]), dict(pair_weight=two), dict(weight=six, d_logprob=six)):
        pref(qn.QNError, **change)
    qn.qn_preference(l, at[:1], two[:0])  # nothing to do
    qn.qn_preference(l[:0], torch.zeros(5, dtype=torch.int64, device="cuda"), two)  # no tokens
    assert torch.allclose(two, torch.full_like(two, math.log(2.0)))
