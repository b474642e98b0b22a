"""Host-only checks of the objectives on a Worker's own answers."""
import ctypes
import math

import pytest
import torch

import objective_reference as ref
import vocab_reference


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import build as qn_build
    from paper_1709_05069_b200 import qn as mod

    qn_build.build()
    mod.lib()
    return mod


def test_bad_arguments_are_refused_before_cuda(qn):
    L, bad = qn.lib(), qn.QN_ERR_INVALID
    host = (ctypes.c_char * 4096)()
    p = ctypes.addressof(host)
    for rows, vocab, dtype, stride, temperature in ((-1, 8, 0, 8, 1.0), (2, 0, 0, 8, 1.0), (2, 8, 5, 8, 1.0), (2, 8, 0, 7, 1.0),
                                                    (2, 8, 0, 8, 0.0), (2, 8, 0, 8, 1.0)):
        # the last one has nothing wrong but that its memory is the host's
        assert L.qn_policy(rows, vocab, dtype, p, stride, p, temperature, p, p, p, p, 0.2, 0.2, 0.0, 0.0, 0.0, p, None, None, None, 0,
                           None) == bad
    assert L.qn_policy(0, 8, 0, None, 8, None, 1.0, None, None, None, None, 0.2, 0.2, 0.0, 0.0, 0.0, None, None, None, None, 0, None) == qn.QN_OK
    for pairs, tokens, dtype, kind, beta in ((-1, 4, 0, 0, 0.1), (1, -1, 0, 0, 0.1), (1, 4, 3, 0, 0.1), (1, 4, 0, 9, 0.1), (1, 4, 0, 0, 0.0),
                                             (1 << 30, 4, 0, 0, 0.1), (1, 4, 0, 0, 0.1)):
        assert L.qn_preference(pairs, tokens, p, dtype, p, p, p, 0, p, kind, beta, 0.0, 0.0, 0, p, p, p, None) == bad
    assert L.qn_preference(0, 4, None, 0, None, None, None, 0, None, 0, 0.1, 0.0, 0.0, 0, None, None, None, None) == qn.QN_OK


def test_binding_refuses_host_tensors(qn):
    z, t, v = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_policy(z, t, v, v.clone(), v.clone())
    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_preference(v, torch.tensor([0, 1, 2]), torch.zeros(1))


def test_reference_gradients_are_those_of_the_reference_losses():
    z = vocab_reference.make_logits(40, 29, torch.float32, 1, device="cpu")
    gen = torch.Generator().manual_seed(2)
    tokens = torch.randint(0, 29, (40,), generator=gen)
    lp = torch.log_softmax(z.double(), 1).gather(1, tokens[:, None])[:, 0]
    old = (lp + 0.3 * torch.randn(40, generator=gen)).float()
    reference, advantage = (lp + 0.5 * torch.randn(40, generator=gen)).float(), torch.randn(40, generator=gen)
    x = z.double().requires_grad_()
    for dual in (0.0, 1.2):
        loss = ref.policy64(x, tokens, old, reference, advantage, None, 1.3, 0.1, 0.2, dual, 0.4, 0.2)[0]
        want, = torch.autograd.grad(loss.sum(), x)
        got = ref.policy64(z, tokens, old, reference, advantage, None, 1.3, 0.1, 0.2, dual, 0.4, 0.2)[3]
        assert torch.allclose(got, want, atol=1e-12)
    lengths = [4, 3, 5, 0]
    at = torch.tensor([1, 5, 8, 13, 13])
    lp, base = -torch.rand(15, dtype=torch.float64, generator=gen), -torch.rand(15, generator=gen)
    w, pw = torch.randint(0, 3, (15,), generator=gen).float(), torch.tensor([0.5, 2.0])
    for kind in (0, 1, 2):
        for normalise in (False, True):
            _, _, grad, _ = ref.preference64(lp, at, base, w, pw, kind, 0.7, 0.1, 0.2, normalise, False)
            for i in range(1, 13):
                both = []
                for h in (1e-6, -1e-6):
                    moved = lp.clone()
                    moved[i] += h
                    both.append((pw * ref.preference64(moved, at, base, w, None, kind, 0.7, 0.1, 0.2, normalise, False)[0]).sum())
                assert abs(float(both[0] - both[1]) / 2e-6 - float(grad[i])) < 1e-7
    assert lengths[3] == 0 and math.isfinite(float(grad[0]))
