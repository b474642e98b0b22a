"""qn_adam_*: constants and states at the ends of what the calls accept, and the ways that an element can take through the step."""
import pytest
import torch

import adam_reference as ref
from test_gpu_adam import BF16, F32, TYPES, Case, qn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("eps,lr,lr_scale,done", [(2.0 ** -126, 1.0, 1.0, 0), (1e-37, 1.0, 1.0, 0), (1.2e-38, 0.5, 64.0, 3),
                                                  (1e-30, 1e9, 1.0, 100), (2.0 ** -126, 1e12, 1.0, 0)])
def test_eps_below_what_a_step_of_the_learning_rate_resolves(qn, bits, offset, eps, lr, lr_scale, done):  # noqa: F811
    """eps / (lr / (1 - beta1^t)) below fp32's normal numbers: elements without history only decay, and those with v = 0 move by
    m' / eps; in whole blocks, alone among ordinary ones, in whole pieces and at ends, on vectors and off them."""
    case = Case(qn, [50, 12_345], F32, F32, False, bits, offset, lr_scale=lr_scale, spread=1.0)
    case.step.fill_(done)
    for i, n in enumerate(case.sizes):
        at = torch.arange(n, device="cuda")
        none = (at % 37 == 0) | ((at // 64) % 5 == 0)
        case.grad[i][none] = 0.0
        for part in (case.m, case.v):
            part[i][none] = 0
        if bits == 8:  # two blocks with m alone: E4M3's 1 at 2^-107
            if n > 900:
                case.m[i][640:704], case.m_scale[i][20:22] = 0x38, 20
                case.v_scale[i][20:22] = 0
        else:
            case.m[i][640:704] = 2.0 ** -107
    case.check_step(lr=lr, eps=eps)
    for part in case.theta:
        assert bool(torch.isfinite(part).all())


@pytest.mark.parametrize("param,grad,master", TYPES)
def test_minus_zero_is_the_same_code_wherever_it_lies(qn, param, grad, master):  # noqa: F811
    """m' = -0, from a code of -0 and gradients that are -0 or vanish beside it: the sign stays, whichever way the neighbours of an
    element need (a root of 0 among them) and wherever the tensor lies."""
    n, runs = 9001, []
    at = torch.arange(n, device="cuda")
    gone = (at % 3 == 1) & ((at // 32) % 2 == 0)
    for offset in (0, 1, 6):
        for apart in (8, 301, n):  # neighbours without history: in every octet, in every warp's elements, one
            case = Case(qn, [n], param, grad, master, 8, offset, 0, seed=6)
            case.m[0][gone] = 0x80
            case.grad[0][gone] = -0.0
            case.grad[0][gone & (at % 2 == 0)] = -1e-45
            lone = (at % apart == 5) & ~gone
            case.v[0][lone], case.grad[0][lone] = 0, 0.0
            qn.qn_adam_step(case.plan, case.step, stochastic=True, seed=2)
            assert bool((case.m[0][gone] == 0x80).all())
            runs.append((apart, case.everything()))
            case.guards_whole()
    for apart, run in runs:
        same = next(x for a, x in runs if a == apart)
        assert all(torch.equal(x, y) for x, y in zip(run, same))


@pytest.mark.parametrize("beta1", [2.0 ** -8 * 0.99, 0.003, 2.0 ** -24 * 1.37, 2.0 ** -30 * 1.7, 2.0 ** -130 * 1.3, 2.0 ** -7 * 1.9,
                                   0.0, 0.5, 0.9, 0.999])
@pytest.mark.parametrize("offset", [0, 1])
def test_small_beta1_and_small_scales(qn, beta1, offset):  # noqa: F811
    """beta1 times a block's power of two may lie below fp32's normal numbers where beta1 times the value that the code stands for does
    not: m' is the latter, in whole pieces and at ends."""
    n = 20_000
    case = Case(qn, [n], F32, F32, False, 8, offset)
    case.grad[0].zero_()
    block = torch.arange((n + 31) // 32, device="cuda")
    case.m_scale[0].copy_(1 + block % 160)
    for seed in (1, 2, 3):
        keep = [x.clone() for x in (case.m[0], case.m_scale[0])]
        case.check_step(beta1=beta1, seed=seed)
        case.m[0].copy_(keep[0])
        case.m_scale[0].copy_(keep[1])


def test_every_root_that_the_packed_way_takes_is_the_correctly_rounded_one(qn):  # noqa: F811
    """All 130 * 2^23 + 1 numbers from 2^-100 to 2^30."""
    def bits(x):
        return int(torch.tensor(x, dtype=F32).view(torch.int32))

    differ = torch.zeros(1, dtype=torch.int64, device="cuda")
    qn.qn_selftest_roots(bits(2.0 ** -100), bits(2.0 ** 30), differ)
    assert int(differ) == 0
    qn.qn_selftest_roots(0, 0, differ)  # the packed way has no root of 0, and this says so
    assert int(differ) == 1
    qn.qn_selftest_roots(0, 6, differ)
    assert 1 < int(differ) <= 8
    for first, last in ((5, 4), (-1, 4), (0, 0x7F800000)):
        with pytest.raises(qn.QNError):
            qn.qn_selftest_roots(first, last, differ)
    with pytest.raises(ValueError):
        qn.qn_selftest_roots(0, 1, differ.cpu())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[0, 40, 0, 3000, 5], [0, 0, 1], [2049, 0], [33, 0, 0, 4100, 0, 0], [0, 9000, 0]])
def test_empty_tensors_among_others(qn, bits, sizes):  # noqa: F811
    """Tensors of no elements before, between and behind others, with 8-bit states too: the others' steps are those of a plan
    without them."""
    some = [n for n in sizes if n]
    alone = Case(qn, some, F32, BF16, False, bits, seed=9)
    beside = Case(qn, some, F32, BF16, False, bits, seed=9)
    nothing = {dtype: torch.empty(0, dtype=dtype, device="cuda") for dtype in (F32, BF16, torch.uint8)}

    def among(part):
        rest = iter(part)
        return [next(rest) if n else nothing[part[0].dtype] for n in sizes]

    scales = dict(m_scale=among(beside.m_scale), v_scale=among(beside.v_scale)) if bits == 8 else {}
    rest = iter(beside.decay)
    sums = [torch.zeros(1, dtype=torch.float64, device="cuda") for _ in range(2)]
    with qn.qn_adam_create(among(beside.theta), among(beside.grad), among(beside.m), among(beside.v), **scales,
                           weight_decay=[next(rest) if n else 0.0 for n in sizes]) as plan:
        assert plan.places == alone.plan.places
        for k in range(2):
            for p, case, sumsq in ((alone.plan, alone, sums[0]), (plan, beside, sums[1])):
                qn.qn_adam_norm(p, sumsq)
                qn.qn_adam_step(p, case.step, sumsq=sumsq, max_norm=0.25, seed=k)
            assert abs(float(sums[0]) / float(sums[1]) - 1) < 1e-12
            sums[1].copy_(sums[0])
            assert all(torch.equal(a, b) for a, b in zip(alone.everything(), beside.everything()))
        values = [[torch.full((plan.places,), 9.0, device="cuda") for _ in range(2)] for _ in range(2)]
        qn.qn_adam_state(alone.plan, *values[0])
        qn.qn_adam_state(plan, *values[1])
        assert all(torch.equal(a, b) for a, b in zip(*values))
    beside.guards_whole()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_tensors_without_gradients_stay_whole(qn, bits, master):  # noqa: F811
    """Parameters, states, scales and master copies of a tensor without a gradient, with others on both sides."""
    case = Case(qn, [40, 3000, 70, 5000], BF16, BF16, master, bits, offset=1, gap=0)
    qn.qn_adam_grads(case.plan, [None if i in (1, 2) else g for i, g in enumerate(case.grad)])
    parts = [p for p in (case.theta, case.master, case.m, case.v, case.m_scale, case.v_scale) if p is not None]
    before = [[p[i].clone() for i in range(4)] for p in parts]
    case.check_step(skip=(1, 2), max_norm=0.01, stochastic=True)
    for p, old in zip(parts, before):
        assert all(torch.equal(p[i], old[i]) for i in (1, 2))
