"""The operators over a vocabulary where a row, a size or an argument is out of the ordinary.

Tolerances are those of test_gpu_vocab.py, which derives them: 5e-6 (1 + |value|) for numbers per row, 1e-5 of the summed
magnitudes of its terms for an element of a gradient, and 2^-8 of it on top where it is stored as bf16.
"""
import math

import pytest
import torch

import vocab_reference as ref
from test_gpu_vocab import DTYPES, check_logprobs, some_tokens

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
