"""qn_adam_*: the AdamW step over many tensors against its 64-bit form; tolerances are derived in adam_reference.step64."""
import math

import pytest
import torch

import adam_reference as ref

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32, False), (F32, BF16, False), (BF16, BF16, False), (BF16, F32, False), (BF16, BF16, True), (BF16, F32, True)]
SIZES = [1, 7, 31, 32, 33, 255, 256, 2047, 2048, 2049, 8191, 20011]


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import qn as mod

    assert torch.cuda.is_available()
    mod.lib()
    return mod


class Case:
    """Tensors in buffers with guard elements between them, their plan, and a 64-bit copy of everything."""

    def __init__(self, qn, sizes, param, grad, master, bits, offset=0, gap=8, seed=1, spread=1e-2, decay=0.1, lr_scale=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.qn, self.sizes, self.bits, self.master_copy = qn, sizes, bits, master
        self.guards = []

        def place(values, dtype, units):
            """One buffer; tensor i at its own place, ``offset`` elements off, with 7s around it."""
            starts, at = [], offset
            for n in units:
                starts.append(at)
                at += n + gap + (-(n + gap)) % 32
            buf = torch.full((at + 32,), 7, dtype=dtype, device="cuda")
            parts = [buf[a:a + n] for a, n in zip(starts, units)]
            for part, x in zip(parts, values):
                part.copy_(x)
            free = torch.ones_like(buf, dtype=torch.bool)
            for a, n in zip(starts, units):
                free[a:a + n] = False
            self.guards.append((buf, free))
            return parts

        def noise(scale):
            return [scale * torch.randn(n, generator=gen, device="cuda") for n in sizes]

        theta, m, root = noise(1.0), noise(0.3 * spread), [x.abs() + 0.1 * spread for x in noise(spread)]
        m[0][0] = 0.0  # a first step's states among them
        root[0][0] = 0.0
        self.theta = place(theta, param, sizes)
        self.master = place([t.float() for t in self.theta], F32, sizes) if master else None
        self.grad = place(noise(spread), grad, sizes)
        blocks = [(n + 31) // 32 for n in sizes]
        self.m_scale = self.v_scale = None
        if bits == 8:
            half = [torch.full((n,), 1 << 15, device="cuda") for n in sizes]
            ms, vs = [ref.scales(x.double()) for x in m], [ref.scales(x.double()) for x in root]
            m = [ref.encode(x.double(), s, h, 3) for x, s, h in zip(m, ms, half)]
            v = [ref.encode(x.double(), s, h, 4) for x, s, h in zip(root, vs, half)]
            self.m_scale, self.v_scale = place(ms, torch.uint8, blocks), place(vs, torch.uint8, blocks)
        else:
            v = [x * x for x in root]
        kind = torch.uint8 if bits == 8 else F32
        self.m, self.v = place(m, kind, sizes), place(v, kind, sizes)
        count = len(sizes)
        self.decay = [decay if i % 3 else 0.0 for i in range(count)]
        self.lr_scale = [lr_scale if i % 2 else 1.0 for i in range(count)]
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        self.plan = qn.qn_adam_create(self.theta, self.grad, self.m, self.v, master=self.master, m_scale=self.m_scale,
                                      v_scale=self.v_scale, weight_decay=self.decay, lr_scale=self.lr_scale)
        self.begin, at = [], 0
        for b in blocks:
            self.begin.append(at)
            at += 32 * b
        assert self.plan.places == at

    def everything(self):
        lists = [self.theta, self.master, self.m, self.v, self.m_scale, self.v_scale]
        return [x.clone() for part in lists if part is not None for x in part] + [self.step.clone()]

    def guards_whole(self):
        for buf, free in self.guards:
            assert bool((buf[free] == 7).all())

    def check_step(self, lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, max_norm=0.0, grad_scale=1.0, stochastic=False, seed=5,
                   skip=(), call=None):
        """One step of the library against the reference, from the states as they are."""
        before = [[x.double() for x in part] if part is not None else None for part in (self.theta, self.master, self.m, self.v)]
        scales = [[x.clone() for x in part] if part is not None else None for part in (self.m_scale, self.v_scale)]
        t = int(self.step) + 1
        sumsq = torch.full((1,), -1.0, dtype=torch.float64, device="cuda")
        squares = sum(float(g.double().square().sum()) for i, g in enumerate(self.grad) if i not in skip)
        if call is None:
            self.qn.qn_adam_norm(self.plan, sumsq)
            self.qn.qn_adam_step(self.plan, self.step, lr=lr, beta1=beta1, beta2=beta2, eps=eps, sumsq=sumsq, max_norm=max_norm,
                                 grad_scale=grad_scale, stochastic=stochastic, seed=seed)
            assert abs(float(sumsq) - squares) <= 1e-12 * squares
        else:
            call()
        assert int(self.step) == t
        c = ref.coefficient(squares, max_norm, grad_scale)
        key = ref.step_key(seed, t)
        for i, n in enumerate(self.sizes):
            theta, master, m0, v0 = (part[i] if part is not None else None for part in before)
            if self.bits == 8:
                m = ref.decode(m0.to(torch.uint8), scales[0][i], 3)
                root = ref.decode(v0.to(torch.uint8), scales[1][i], 4)
                v = ref.f32(root * root)
            else:
                m, v = m0, v0
            if i in skip:
                assert torch.equal(self.theta[i].double(), theta) and torch.equal(self.m[i].double(), m0)
                assert torch.equal(self.v[i].double(), v0)
                continue
            g = self.grad[i].double()
            want, m1, v1, theta_off, m_off, v_off = ref.step64(theta if master is None else master, g, m, v, t, lr * self.lr_scale[i],
                                                               beta1, beta2, eps, self.decay[i], c)
            place = self.begin[i] + torch.arange(n, device="cuda")
            word = ref.words(key, place)
            if self.bits == 8:
                m32, r32 = ref.moments32(m, v, g, beta1, beta2, c)
                ms, vs = ref.scales(m32), ref.scales(r32)
                assert torch.equal(self.m_scale[i], ms) and torch.equal(self.v_scale[i], vs)
                assert torch.equal(self.m[i], ref.encode(m32, ms, word >> 16, 3))
                assert torch.equal(self.v[i], ref.encode(r32, vs, word & 65535, 4))
                # and, apart from how codes are chosen, they are within one step of the moving averages
                got_m, got_r = ref.decode(self.m[i], ms, 3), ref.decode(self.v[i], vs, 4)
                step_m = m1.abs() / 8 + 2.0 ** (ref.each(ms, n).double() - 127 - 9)
                step_r = v1.sqrt() / 16 + 2.0 ** (ref.each(vs, n).double() - 127 - 10)
                assert bool(((got_m - m1).abs() <= step_m * 1.001 + m_off).all())
                # the root lies between those of v' - v_off and v' + v_off; that is 5 ulp of it for ordinary numbers, and far more below
                # 2^-126, where v' has steps of 2^-149: 3e-5 of v' = 5e-41
                spread = (v1 + v_off).sqrt() - (v1 - v_off).clamp(min=0.0).sqrt()
                assert bool(((got_r - v1.sqrt()).abs() <= step_r * 1.001 + spread + 2 * ref.ULP * v1.sqrt()).all())
            else:
                assert bool(((self.m[i].double() - m1).abs() <= m_off).all())
                assert bool(((self.v[i].double() - v1).abs() <= v_off).all())
            got = self.theta[i].double()
            if master is not None:
                assert bool(((self.master[i].double() - want).abs() <= theta_off).all())
                assert torch.equal(self.theta[i], self.master[i].to(BF16))
            elif self.theta[i].dtype == F32:
                assert bool(((got - want).abs() <= theta_off).all())
            else:  # half a step of bf16, or a whole one by chance
                assert bool(((got - want).abs() <= theta_off + want.abs() * (2.0 ** -7 if stochastic else 2.0 ** -8)).all())
        self.guards_whole()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("offset,gap", [(0, 8), (0, 0), (1, 3), (5, 0)])
def test_step_of_many_tensors(qn, param, grad, master, bits, offset, gap):
    case = Case(qn, SIZES, param, grad, master, bits, offset, gap, lr_scale=0.5)
    for k in range(3):
        case.check_step(max_norm=(0.0, 0.5, 1e6)[k], grad_scale=(1.0, 0.25, -2.0)[k], stochastic=k == 1)
        for g in case.grad:
            g.copy_(torch.flip(g, (0,)) * 0.5)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta1,beta2,eps,lr", [(0.0, 0.0, 1e-8, 1e-2), (0.9, 0.999, 1e-6, 0.0), (0.99, 0.9999, 1e-3, 1.0)])
def test_other_rates(qn, bits, beta1, beta2, eps, lr):
    case = Case(qn, [1, 100, 4099], F32, F32, False, bits)
    case.step.fill_(10)
    case.check_step(lr=lr, beta1=beta1, beta2=beta2, eps=eps)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", TYPES)
def test_one_large_tensor_among_small_ones(qn, param, grad, master, bits):
    """Enough pieces for every CTA to come round several times."""
    case = Case(qn, [3, 9_000_001, 64, 1_000_000], param, grad, master, bits, spread=1.0)
    case.check_step(max_norm=1.0, stochastic=True, seed=(1 << 40) + 3)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zeros_moves_by_the_learning_rate(qn, bits):
    """m' / sqrt(v') is the gradient's sign on the first step, whatever its size; 0 stays."""
    n = 1000
    g = torch.randn(n, device="cuda") * torch.logspace(-12, 6, n, device="cuda")
    g[::10] = 0.0
    case = Case(qn, [n], F32, F32, False, bits, decay=0.0)
    for part in (case.theta, case.m, case.v, case.m_scale, case.v_scale):
        if part is not None:
            part[0].zero_()
    case.grad[0].copy_(g)
    qn.qn_adam_step(case.plan, case.step, lr=0.125, eps=1e-30)
    assert torch.allclose(case.theta[0], -0.125 * torch.sign(g), rtol=1e-5, atol=0)
    if bits == 8:  # no root is lost, however small beside its block's largest
        assert bool(((case.v[0] > 0) == (g != 0)).all())


def test_codes_keep_the_mean_where_a_step_is_smaller_than_a_code(qn):
    """Roots that fall by 1/2000 a step, codes 1/16 apart: after 400 steps without gradient the mean of 2^16 elements has
    fallen as it should.  Each step's rounding has a variance of 1/4 of a code's step at most: 400 of them leave a standard
    error of the mean of 0.5 sqrt(400) / 256 / 16 = 0.0025 relative; six of these are allowed."""
    n = 1 << 16
    case = Case(qn, [n], F32, F32, False, 8, decay=0.0)
    root = 1.0 + 0.9 * torch.rand(n, device="cuda")
    case.v_scale[0].copy_(ref.scales(root.double()))
    case.v[0].copy_(ref.encode(root.double(), case.v_scale[0], torch.full((n,), 1 << 15, device="cuda"), 4))
    case.m[0].copy_(case.v[0] >> 1)  # the same numbers with one bit less
    case.m_scale[0].copy_(case.v_scale[0])
    case.grad[0].zero_()
    start_m, start_r = ref.decode(case.m[0], case.m_scale[0], 3).mean(), ref.decode(case.v[0], case.v_scale[0], 4).mean()
    for _ in range(400):
        qn.qn_adam_step(case.plan, case.step, lr=0.0, beta1=0.999, beta2=0.999, seed=77)
    end_m, end_r = ref.decode(case.m[0], case.m_scale[0], 3).mean(), ref.decode(case.v[0], case.v_scale[0], 4).mean()
    assert abs(float(end_m / start_m) / 0.999 ** 400 - 1) < 6 * 0.005 / 0.999 ** 400
    assert abs(float(end_r / start_r) / 0.999 ** 200 - 1) < 6 * 0.0025 / 0.999 ** 200


def test_bf16_parameters_rounded_by_chance_keep_the_mean(qn):
    """Steps of 2^-12 on parameters of 1.25, whose steps are 2^-7: to nearest nothing moves, by chance the mean does.  64 steps of
    a variance of 2^-16 at most over 2^16 elements: a standard error of 8 * 2^-8 / 256; six are allowed."""
    n = 1 << 16
    for stochastic in (False, True):
        case = Case(qn, [n], BF16, F32, False, 32, decay=0.0)
        case.theta[0].fill_(1.25)
        case.m[0].zero_()
        case.v[0].zero_()
        case.grad[0].fill_(1.0)
        for _ in range(64):
            qn.qn_adam_step(case.plan, case.step, lr=2.0 ** -12, eps=1e-12, stochastic=stochastic, seed=3)
        mean = float(case.theta[0].double().mean())
        assert mean == 1.25 if not stochastic else abs(mean - (1.25 - 64 * 2.0 ** -12)) < 6 * 8 * 2.0 ** -8 / 256


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_gradients_that_are_not_finite(qn, bits, bad):
    case = Case(qn, [100, 5000], F32, BF16, False, bits)
    case.grad[1][4321] = bad
    before, sumsq = case.everything(), torch.zeros(1, dtype=torch.float64, device="cuda")
    qn.qn_adam_norm(case.plan, sumsq)
    assert not math.isfinite(float(sumsq))
    for max_norm in (0.0, 1.0):
        qn.qn_adam_step(case.plan, case.step, sumsq=sumsq, max_norm=max_norm)
        assert all(torch.equal(a, b) for a, b in zip(before, case.everything()))
    # without the norm they reach their own element and no other
    qn.qn_adam_step(case.plan, case.step)
    assert int(case.step) == 1
    assert bool(torch.isfinite(case.theta[0]).all()) and int((~torch.isfinite(case.theta[1])).sum()) == (1 if bad != bad else 1)
    if bits == 8:
        m = ref.decode(case.m[1], case.m_scale[1], 3)
        assert bool(torch.isnan(m[4321])) and int(torch.isnan(m).sum()) == 1 and int(case.v[1][4321]) == 255
    # and the next step with ordinary ones works from what is there
    case.grad[1][4321] = 0.5
    case.grad[0].zero_()
    qn.qn_adam_step(case.plan, case.step)
    assert int(case.step) == 2 and bool(torch.isfinite(case.theta[0]).all())
    case.guards_whole()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("offset", [1, 6, 11])
def test_results_do_not_depend_on_where_tensors_lie(qn, param, grad, master, bits, offset):
    """The same bits on vectors and off them, in whole pieces too, with elements of every kind among them."""
    runs = []
    for off in (0, offset):
        case = Case(qn, [30_000, 40, 9001, 2049], param, grad, master, bits, off, 0, seed=4)
        for g in case.grad[::2]:
            g[5::1031], g[6::2077], g[2500::4099], g[33::67] = 0.0, 1e20, 1e-30, 1e-12
        case.grad[0][12_000], case.grad[0][12_700], case.grad[0][20_001] = math.inf, math.nan, -math.inf
        case.theta[0][13_500], case.theta[0][14_001] = math.nan, math.inf
        if master:
            case.master[0][13_500], case.master[0][14_001] = math.nan, math.inf
        if bits == 8:  # a block without history
            for state in (case.m, case.m_scale, case.v, case.v_scale):
                state[0][: 480 if state is case.m or state is case.v else 15] = 0
            for x, n in ((case.m, 9600), (case.v, 9600)):
                x[0][9000:n] = 0
        for k in range(3):
            qn.qn_adam_step(case.plan, case.step, lr=1e-2, stochastic=True, seed=k)
        runs.append(case.everything())
        case.guards_whole()
    for a, b in zip(*runs):
        assert bool(((a == b) | ((a != a) & (b != b))).all())


@pytest.mark.parametrize("param,grad,master", TYPES)
@pytest.mark.parametrize("offset", range(1, 16))
def test_codes_wherever_they_lie(qn, param, grad, master, offset):
    """Every place within a vector, in tensors with whole pieces inside."""
    case = Case(qn, [9001, 40, 16_385], param, grad, master, 8, offset, 0, seed=offset)
    for k in range(2):
        case.check_step(stochastic=k == 1)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("repeats,each,offset", [(1, 32, 0), (16, 32, 0), (16, 32, 1), (60, 8, 0), (60, 8, 3), (25, 256, 0)])
def test_extreme_gradients(qn, bits, repeats, each, offset):
    """The least and the largest fp32 numbers beside ordinary ones, at the ends of the scales' range: in blocks of their own,
    side by side in a block, and in blocks of zeros, in pieces that end and in whole ones."""
    values = [0.0, 1e-45, 1e-38, 1.2e-38, 1e-20, 1e-6, 1.0, 1e6, 1e15, 1e19, -1e19, 3e18]
    n = each * len(values) * repeats
    case = Case(qn, [n], F32, F32, False, bits, offset)
    g = torch.tensor(values, device="cuda").repeat_interleave(each).repeat(repeats)
    if each != 256:
        g[::7] = 1e-3
    case.grad[0].copy_(g)
    for part in (case.m, case.v, case.m_scale, case.v_scale):
        if part is not None:
            part[0].zero_()
    for _ in range(2):
        case.check_step(beta1=0.5, beta2=0.5)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("param,grad,master", TYPES)
def test_numbers_that_are_not_finite_stay_in_their_places(qn, param, grad, master, offset):
    """Infinite and NaN gradients, and parameters that are NaN already, in whole pieces and at ends: every other element is what it is
    without them, but that codes of a block follow its scale."""
    n = 9001
    bad = [0, 100, 2047, 2048, 4100, 8191, 8999]
    runs = []
    for spoil in (False, True):
        case = Case(qn, [n], param, grad, master, 8, offset)
        if spoil:
            case.grad[0][bad[:3]] = math.inf
            case.grad[0][bad[3:5]] = math.nan
            (case.master or case.theta)[0][bad[5:]] = math.nan
        qn.qn_adam_step(case.plan, case.step, stochastic=True, seed=8)
        case.guards_whole()
        runs.append(case)
    hit = torch.zeros(n, dtype=torch.bool, device="cuda")
    hit[bad] = True
    theta, want = runs[1].theta[0], runs[0].theta[0]
    assert bool(torch.isnan(theta[hit]).all()) and torch.equal(theta[~hit], want[~hit])
    m = ref.decode(runs[1].m[0], runs[1].m_scale[0], 3)
    assert torch.isnan(m).nonzero()[:, 0].tolist() == bad[:5]
    block = torch.zeros((n + 31) // 32, dtype=torch.bool, device="cuda")
    block[torch.tensor(bad[:5], device="cuda") // 32] = True
    elsewhere = ~block.repeat_interleave(32)[:n]
    assert torch.equal(runs[1].m[0][elsewhere], runs[0].m[0][elsewhere]) and torch.equal(runs[1].v[0][elsewhere], runs[0].v[0][elsewhere])


@pytest.mark.parametrize("bits,offset", [(32, 0), (8, 0), (8, 1)])
def test_steps_in_a_row_are_those_one_by_one(qn, bits, offset):
    """Launches whose set-up overlaps the end of the last one read what that has written."""
    runs = []
    for wait in (True, False):
        case = Case(qn, [1_500_001, 33, 700_000], BF16, BF16, False, bits, offset)
        sumsq = torch.zeros(1, dtype=torch.float64, device="cuda")
        for _ in range(40):
            qn.qn_adam_norm(case.plan, sumsq)
            if wait:
                torch.cuda.synchronize()
            qn.qn_adam_step(case.plan, case.step, sumsq=sumsq, max_norm=1.0, stochastic=True, seed=4)
            if wait:
                torch.cuda.synchronize()
        runs.append(case.everything())
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_many_small_tensors(qn):
    sizes = [1 + (37 * i) % 90 for i in range(1500)]
    for bits in (32, 8):
        case = Case(qn, sizes, F32, F32, False, bits, offset=1, gap=0)
        qn.qn_adam_grads(case.plan, [g.clone() for g in case.grad])
        qn.qn_adam_grads(case.plan, case.grad)
        case.check_step(max_norm=0.1)


def test_tensors_without_gradients_and_empty_ones(qn):
    for bits in (32, 8):
        case = Case(qn, [0, 40, 0, 3000, 5] if bits == 32 else [1, 40, 2, 3000, 5], F32, F32, False, bits) if bits == 8 else \
            Case(qn, [64, 40, 7, 3000, 5], F32, F32, False, bits)
        qn.qn_adam_grads(case.plan, [None if i in (1, 3) else g for i, g in enumerate(case.grad)])
        case.check_step(skip=(1, 3), max_norm=0.01)
        moved = [g.clone() for g in case.grad]
        for g in case.grad:
            g.fill_(math.nan)
        qn.qn_adam_grads(case.plan, moved)
        old, case.grad = case.grad, moved
        case.check_step()
        del old


def test_empty_tensors(qn):
    empty, n = torch.empty(0, device="cuda"), 50
    theta, g, m, v = torch.ones(n, device="cuda"), torch.ones(n, device="cuda"), torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    step, sumsq = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.ones(1, dtype=torch.float64, device="cuda")
    with qn.qn_adam_create([empty, theta, empty], [empty, g, None], [empty, m, empty], [empty, v, empty]) as plan:
        qn.qn_adam_norm(plan, sumsq)
        qn.qn_adam_step(plan, step, lr=0.5, sumsq=sumsq)
        assert float(sumsq) == n and torch.allclose(theta, torch.full_like(theta, 0.5)) and plan.places == 64
    with qn.qn_adam_create([empty], [None], [empty], [empty]) as plan:  # nothing at all
        qn.qn_adam_norm(plan, sumsq)
        qn.qn_adam_step(plan, step, sumsq=sumsq, max_norm=1.0)
        qn.qn_adam_state(plan, empty, empty)
        assert float(sumsq) == 0.0 and int(step) == 2


def test_learning_rate_on_the_device_and_seeds(qn):
    runs = []
    for lr, seed in ((1e-3, 1), (torch.tensor([1e-3], device="cuda"), 1), (1e-3, 2), (1e-3, 1 + (1 << 32))):
        case = Case(qn, [5000], BF16, F32, False, 8)
        if not isinstance(lr, torch.Tensor):
            lr = float(torch.tensor(lr, dtype=F32))
        for _ in range(3):
            qn.qn_adam_step(case.plan, case.step, lr=lr, stochastic=True, seed=seed)
        runs.append(case.everything())
    same = [all(torch.equal(a, b) for a, b in zip(runs[0], r)) for r in runs]
    assert same == [True, True, False, False]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("offset", range(8))
def test_what_codes_stand_for_wherever_they_lie(qn, offset, dtype):
    """Every place of a tensor's first code within a vector, the smallest sizes, and pieces' ends."""
    sizes = [1, 3, 7, 8, 9, 11, 12, 13, 20, 31, 33, 2047, 2048, 2049, 2060, 70_001]
    case = Case(qn, sizes, F32, BF16, False, 8, offset=offset, gap=1, seed=offset)
    m, root = (torch.full((case.plan.places,), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    qn.qn_adam_state(case.plan, m, root)
    for got, codes, scales, bits in ((m, case.m, case.m_scale, 3), (root, case.v, case.v_scale, 4)):
        want = torch.zeros_like(got)
        for i, n in enumerate(sizes):
            want[case.begin[i]:case.begin[i] + n] = ref.decode(codes[i], scales[i], bits).to(dtype)
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bits", [32, 8])
def test_what_states_stand_for(qn, bits, dtype):
    case = Case(qn, [33, 1, 5000, 64], F32, F32, False, bits, offset=1, gap=3)
    m, root = (torch.full((case.plan.places,), 9.0, dtype=dtype, device="cuda") for _ in range(2))
    qn.qn_adam_state(case.plan, m, root)
    end = case.plan.places
    for i in reversed(range(4)):
        n, at = case.sizes[i], case.begin[i]
        if bits == 8:
            want = ref.decode(case.m[i], case.m_scale[i], 3), ref.decode(case.v[i], case.v_scale[i], 4)
        else:
            want = case.m[i].double(), ref.f32(case.v[i].double().sqrt())
        for got, x in zip((m, root), want):
            assert torch.equal(got[at:at + n], x.to(dtype)) and not bool(got[at + n:end].any())
        end = at
    again = torch.zeros_like(m)
    qn.qn_adam_state(case.plan, again, None)
    assert torch.equal(again, m)
    case.guards_whole()


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_steps_are_those_of_eager_calls(qn, bits):
    """Norm and step in one graph on another stream, with the step's count, the norm and the learning rate on the device."""
    eager, graphed = (Case(qn, SIZES, BF16, BF16, False, bits) for _ in range(2))
    lr, sumsq = torch.tensor([1e-2], device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")

    def both(case):
        qn.qn_adam_norm(case.plan, sumsq)
        qn.qn_adam_step(case.plan, case.step, lr=lr, sumsq=sumsq, max_norm=0.1, stochastic=True, seed=9)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both(graphed)
    assert int(graphed.step) == 0
    for k in range(4):
        lr.fill_(1e-2 / (k + 1))
        for case in (eager, graphed):
            for g in case.grad:
                g.mul_(0.9)
        both(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager.everything(), graphed.everything()))


def test_plans_on_two_streams_at_once(qn):
    cases, wants = [Case(qn, [300_000, 77], F32, F32, False, 8, seed=s) for s in (1, 2)], []
    for s in (1, 2):
        alone = Case(qn, [300_000, 77], F32, F32, False, 8, seed=s)
        for _ in range(20):
            qn.qn_adam_step(alone.plan, alone.step)
        wants.append(alone.everything())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(20):
        for case, stream in zip(cases, streams):
            qn.qn_adam_step(case.plan, case.step, stream=stream)
    torch.cuda.synchronize()
    for case, want in zip(cases, wants):
        assert all(torch.equal(a, b) for a, b in zip(case.everything(), want))


def test_elements_past_2_to_the_31(qn):
    n = (1 << 31) + 70
    theta, g = torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n, dtype=BF16, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    ms, vs = (torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    step, sumsq = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    at = torch.tensor([0, 1 << 30, (1 << 31) - 1, 1 << 31, (1 << 31) + 63, n - 1], device="cuda")
    g[at] = torch.tensor([1.0, -2.0, 3.0, -4.0, 5.0, -6.0], dtype=BF16, device="cuda")
    with qn.qn_adam_create([theta], [g], [m], [v], m_scale=[ms], v_scale=[vs]) as plan:
        qn.qn_adam_norm(plan, sumsq)
        qn.qn_adam_step(plan, step, lr=0.5, sumsq=sumsq, eps=1e-20)
        assert float(sumsq) == 91.0
        assert torch.equal(theta[at], (-0.5 * torch.sign(g[at])).to(BF16))
        assert int((theta != 0).sum()) == len(at) == int((v != 0).sum()) == int((m != 0).sum())
        word = ref.words(ref.step_key(0, 1), at)
        root = ref.f32(torch.sqrt(ref.f32(ref.f32(g[at].double() ** 2) * ref.f32(1.0 - 0.999))))
        block = vs[at // 32]
        assert torch.equal(vs[at // 32], ((torch.frexp(root).exponent - 8) + 127).to(torch.uint8))
        y = root * 2.0 ** (127.0 - block.double())
        assert torch.equal(v[at], (torch.floor(y / 8 + ((word & 65535).double() + 0.5) / 65536) - 16 + 16 * 14).to(torch.uint8))


# ---- refusals ------------------------------------------------------------------------------------------------------------


def test_refusals(qn):
    n = 64
    new = lambda dtype=F32, size=n: torch.zeros(size, dtype=dtype, device="cuda")  # noqa: E731
    theta, g, m, v = new(), new(), new(), new()
    codes, few = new(torch.uint8), new(torch.uint8, 2)
    good = dict(params=[theta], grads=[g], m=[m], v=[v])

    def refused(match, kind=ValueError, **change):
        with pytest.raises(kind, match=match):
            qn.qn_adam_create(**{**good, **change})

    refused("params must be", params=[])
    refused("params must be", params=[theta.cpu()])
    refused("storage dtype", kind=TypeError, params=[theta.half()])
    refused("storage dtype", kind=TypeError, grads=[g.half()])
    refused("grads must be", grads=[g.cpu()])
    refused("grads must be", grads=[new(size=n + 1)])
    refused("grads must be", grads=[new(size=2 * n)[::2]])
    refused("grads must be a list", grads=[])
    refused("grads must be a list", grads=g)
    refused("m must be", m=[m.to(BF16)])
    refused("v must be", v=[codes])
    refused("m must be", m_scale=[few], v_scale=[few.clone()])
    refused("m_scale must be", m=[codes], v=[codes.clone()], m_scale=[new(torch.uint8, 3)], v_scale=[few])
    refused("invalid|bad", kind=qn.QNError, m=[codes], v=[codes.clone()], m_scale=[few])
    refused("invalid|bad", kind=qn.QNError, m=[None])
    refused("invalid|bad", kind=qn.QNError, master=[new()])  # parameters are fp32 already
    refused("invalid|bad", kind=qn.QNError, weight_decay=-1.0)
    refused("invalid|bad", kind=qn.QNError, lr_scale=math.nan)
    refused("invalid|bad", kind=qn.QNError, m=[theta])  # the same memory twice
    refused("invalid|bad", kind=qn.QNError, grads=[theta])
    two = new(size=n + 1)
    refused("invalid|bad", kind=qn.QNError, params=[two[:n]], m=[two[1:]])
    refused("invalid|bad", kind=qn.QNError, params=[theta, theta], grads=[g, g], m=[m, new()], v=[v, new()])
    # one gradient for two tensors is read only
    qn.qn_adam_create([theta, new()], [g, g], [m, new()], [v, new()]).close()
    step, sumsq = new(torch.int64, 1), new(torch.float64, 1)
    with qn.qn_adam_create(**good) as plan:
        for change in (dict(lr=-1.0), dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=1e-60),
                       dict(max_norm=1.0), dict(max_norm=math.nan), dict(grad_scale=math.inf)):
            with pytest.raises(qn.QNError):
                qn.qn_adam_step(plan, step, **change)
        for bad in (step.cpu(), step.int(), new(torch.int64, 2)):
            with pytest.raises(ValueError, match="step must be"):
                qn.qn_adam_step(plan, bad)
        with pytest.raises(ValueError, match="lr must be"):
            qn.qn_adam_step(plan, step, lr=new(torch.float64, 1))
        with pytest.raises(ValueError, match="sumsq must be"):
            qn.qn_adam_norm(plan, sumsq.float())
        with pytest.raises(qn.QNError):
            qn.qn_adam_grads(plan, [m])
        with pytest.raises(ValueError):
            qn.qn_adam_grads(plan, [g.to(BF16)])
        with pytest.raises(qn.QNError):
            qn.qn_adam_state(plan, m, None)
        both = new(size=n + 1)
        with pytest.raises(qn.QNError):
            qn.qn_adam_state(plan, both[:n], both[1:])
        assert int(step) == 0 and not bool(theta.any())
    plan.close()  # once more is nothing
    L = qn.lib()
    assert L.qn_adam_step(None, step.data_ptr(), 1e-3, None, 0.9, 0.99, 1e-8, None, 0.0, 1.0, 0, 0, None) == qn.QN_ERR_INVALID
