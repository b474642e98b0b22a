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
