"""The gradient calls where every cluster of CTAs takes many rows, one after the other, with padding between them: against
the 64-bit forms, block of rows by block of rows.  Tolerances as in test_gpu_vocab.py.

The sizes stand for cluster sizes of 1, 2, 5 and 8 CTAs (148, 74, about 28 and about 15 clusters on the device), for more
rows than twice the six that a cluster has under way at a time, and for the three forms of a row: on 16 bytes, elsewhere, and
with its gradient elsewhere again.
"""
import math

import pytest
import torch

import vocab_reference as ref
from test_gpu_vocab import close

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
# dtype, rows, vocab, elements between rows and before the first of them, the same of the gradient
ALIGNED = [(BF16, 2100, 16896, 0, 0, 0, 0), (F32, 2100, 8448, 0, 0, 0, 0), (BF16, 1000, 131072, 8, 0, 8, 0),
           (F32, 1000, 65536, 0, 0, 0, 0), (BF16, 400, 300000, 0, 0, 0, 0), (F32, 220, 262144, 0, 0, 0, 0)]
EDGES = [(BF16, 2100, 33001, 0, 0, 0, 0), (F32, 2100, 16411, 2, 3, 2, 3), (BF16, 1100, 70001, 7, 1, 7, 1),
         (F32, 420, 95003, 0, 2, 0, 2), (BF16, 220, 300001, 0, 5, 0, 5), (F32, 220, 150001, 1, 0, 1, 0)]
ELSEWHERE = [(BF16, 2100, 33001, 0, 0, 7, 0), (F32, 2100, 16411, 0, 0, 0, 1), (BF16, 1100, 70001, 0, 0, 2, 3),
             (F32, 420, 95003, 1, 0, 2, 0), (BF16, 220, 300000, 0, 0, 0, 1), (F32, 220, 150001, 0, 1, 0, 0)]


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import qn as mod

    assert torch.cuda.is_available()
    mod.lib()
    return mod


def matrix(dtype, rows, vocab, pad, offset, fill=None):
    store = torch.empty(offset + rows * (vocab + pad) + 8, dtype=dtype, device="cuda")
    if fill is not None:
        store.fill_(fill)
    return store.as_strided((rows, vocab), (vocab + pad, 1), offset)


def tokens_of(rows, vocab, k, gen):
    """k different tokens a row: spread over it, or side by side; some rows have the first or the last of all."""
    start = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    start[::5] = 0
    start[1::5] = vocab - 1
    step = torch.where(torch.arange(rows, device="cuda") % 2 == 0, vocab // k, 1)
    return (start[:, None] + step[:, None] * torch.arange(k, device="cuda")) % vocab


def blocks(rows, vocab):
    size = max(1, (1 << 24) // vocab)
    return [slice(a, min(a + size, rows)) for a in range(0, rows, size)]


def check_gradient(out, z, want_of):
    for b in blocks(*z.shape):
        want, bound = want_of(b)
        bound = bound + 1e-30
        if z.dtype == BF16:
            bound = bound + 2.0 ** -8 * want.abs() + 2.0 ** -133
        close(out[b], want, bound, b)


def same_bits(a, b):
    kind = torch.int16 if a.dtype == BF16 else torch.int32
    return torch.equal(a.view(kind), b.view(kind))


def case(shape, seed):
    dtype, rows, vocab, pad, offset, out_pad, out_offset = shape
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = matrix(dtype, rows, vocab, pad, offset)
    z.normal_(0.0, 3.0, generator=gen)
    padding = torch.zeros(rows, dtype=torch.bool, device="cuda")
    padding[1::3] = True
    padding[rows // 2:rows // 2 + 40] = False
    z[padding] = math.nan
    z[::7, ::2] = -math.inf
    z[5] = -math.inf
    in_place = matrix(dtype, rows, vocab, pad, offset)
    in_place.copy_(z)
    return z, matrix(dtype, rows, vocab, out_pad, out_offset, 7.0), in_place, padding, gen


@pytest.mark.parametrize("entropy", [False, True])
@pytest.mark.parametrize("shape", ALIGNED + EDGES + ELSEWHERE)
def test_backward_over_many_rows(qn, shape, entropy):
    z, out, in_place, padding, gen = case(shape, 1)
    rows, vocab = z.shape
    k, temperature = 9, 0.9
    top = tokens_of(rows, vocab, k, gen)
    top[3::11, 4:] = -1
    t = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
    t[2::9] = -1

    def upstream(*shape_):
        return torch.randn(shape_, generator=gen, device="cuda").masked_fill(
            padding[:, None] if len(shape_) == 2 else padding, 0.0)

    g, gh, gt = upstream(rows), upstream(rows) if entropy else None, upstream(rows, k)
    for src, dst in ((z, out), (in_place, in_place)):
        qn.qn_logprobs_backward(src, dst, tokens=t, d_logprob=g, d_entropy=gh, top_token=top, d_top_logprob=gt,
                                temperature=temperature)

    def want_of(b):
        want, size = ref.backward64(z[b], t[b], temperature, g[b], None, gh[b] if entropy else None, top[b], gt[b])
        return want, 1e-5 * torch.where(padding[b, None], 0.0, size)

    check_gradient(out, z, want_of)
    check_gradient(in_place, z, want_of)
    # a gradient that lies elsewhere may be shared out over another number of CTAs, and be added up in another order
    assert shape in ELSEWHERE or same_bits(out, in_place)


@pytest.mark.parametrize("logprobs", [False, True])
@pytest.mark.parametrize("shape", ALIGNED + EDGES + ELSEWHERE)
def test_distill_over_many_rows(qn, shape, logprobs):
    z, out, in_place, padding, gen = case(shape, 2)
    rows, vocab = z.shape
    k, temperature = 40, 1.6
    token = tokens_of(rows, vocab, k, gen)
    value = torch.log_softmax(2.0 * torch.randn((rows, k + 1), generator=gen, device="cuda"), 1)[:, :k].contiguous()
    token[4::11, 7:] = -1
    token[13] = -1
    w = (torch.rand(rows, generator=gen, device="cuda") + 0.5).masked_fill(padding, 0.0)
    mode = qn.QN_TEACHER_LOGPROBS if logprobs else qn.QN_TEACHER_LOGITS
    loss, again, alone = (torch.full((rows,), 9.0, device="cuda") for _ in range(3))
    qn.qn_distill(z, token, value, alone, weight=w, temperature=temperature, teacher=mode)
    for src, dst, to in ((z, out, loss), (in_place, in_place, again)):
        qn.qn_distill(src, token, value, to, dlogits=dst, weight=w, temperature=temperature, teacher=mode)

    def want_of(b):
        want, grad, loss_size, size, slack = ref.distill64(z[b], token[b], value[b], logprobs, temperature, w[b])
        for x in (loss, again, alone):
            close(x[b], want, 5e-6 * (1 + loss_size.nan_to_num(0, 0, 0)), ("loss", b))
        return grad, torch.where(padding[b, None], 0.0, 1e-5 * size + 1e-6 * slack)

    check_gradient(out, z, want_of)
    check_gradient(in_place, z, want_of)
    assert shape in ELSEWHERE or same_bits(out, in_place) and same_bits(loss, again)


@pytest.mark.parametrize("shape", [ALIGNED[2], ALIGNED[3], ALIGNED[5], EDGES[2], EDGES[5]])
def test_loss_alone_over_many_rows_is_the_same_each_time(qn, shape):
    """Without a gradient a part of a row is given back as soon as it has been added, and the warps run far ahead of one
    another: none may take a place in shared memory before its copy has come."""
    z, _, _, padding, gen = case(shape, 3)
    rows, vocab = z.shape
    token = tokens_of(rows, vocab, 8, gen)
    value = torch.log_softmax(torch.randn((rows, 9), generator=gen, device="cuda"), 1)[:, :8].contiguous()
    w = torch.ones(rows, device="cuda").masked_fill(padding, 0.0)
    losses = torch.full((60, rows), 9.0, device="cuda")
    for loss in losses:
        qn.qn_distill(z, token, value, loss, weight=w)
    for b in blocks(rows, vocab):
        want, _, size, _, _ = ref.distill64(z[b], token[b], value[b], True, 1.0, w[b])
        close(losses[0, b], want, 5e-6 * (1 + size.nan_to_num(0, 0, 0)), b)
    assert all(same_bits(losses[0], loss) for loss in losses)
