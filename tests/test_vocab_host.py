"""Host-only checks of the operators over a vocabulary: no GPU is needed to be refused."""
import ctypes

import pytest
import torch


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
    for rows, vocab, dtype, stride, temperature in ((-1, 8, 0, 8, 1.0), (2, 0, 0, 8, 1.0), (2, 8, 5, 8, 1.0),
                                                    (2, 8, 0, 7, 1.0), (2, 8, 0, 8, 0.0), (2, 8, 0, 8, float("nan")),
                                                    (2, 1 << 31, 0, 1 << 31, 1.0), (2, 8, 0, 8, 1.0)):
        # the last one has nothing wrong but that its memory is the host's
        assert L.qn_logprobs(rows, vocab, dtype, p, stride, p, temperature, p, p, p, 0, None, None, None) == bad
        assert L.qn_logprobs_backward(rows, vocab, dtype, p, stride, p, temperature, p, None, None, 0, None, None, p,
                                      stride, None) == bad
        assert L.qn_distill(rows, vocab, dtype, p, stride, 2, p, 0, p, 1, temperature, None, p, None, 0, None) == bad
    assert L.qn_logprobs(2, 8, 0, None, 8, p, 1.0, p, p, p, 0, None, None, None) == bad


def test_nothing_to_do_is_no_error(qn):
    L = qn.lib()
    assert L.qn_logprobs(0, 8, 0, None, 8, None, 1.0, None, None, None, 0, None, None, None) == qn.QN_OK
    assert L.qn_logprobs_backward(0, 8, 0, None, 8, None, 1.0, None, None, None, 0, None, None, None, 8, None) == qn.QN_OK
    assert L.qn_distill(0, 8, 0, None, 8, 2, None, 0, None, 1, 1.0, None, None, None, 0, None) == qn.QN_OK


def test_binding_refuses_host_tensors(qn):
    z, t, v = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), torch.zeros(2)
    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_logprobs(z, t, v)
    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_logprobs_backward(z, z.clone(), tokens=t, d_logprob=v)
    with pytest.raises(ValueError, match="CUDA tensor"):
        qn.qn_distill(z, t.view(2, 1), v.view(2, 1), v)


def test_reference_gradients_are_those_of_the_reference_losses():
    """The 64-bit forms that the GPU tests compare with, against torch's own derivative of the loss."""
    import vocab_reference as ref

    z = ref.make_logits(3, 29, torch.float32, 1, device="cpu").double().requires_grad_()
    for logprobs in (False, True):
        top = (z.detach() + torch.randn(3, 29, dtype=torch.float64)).topk(5, 1)
        value = (top.values - 4.5) if logprobs else top.values
        loss, grad, *_ = ref.distill64(z, top.indices, value, logprobs, 1.3, None)
        want, = torch.autograd.grad(loss.sum(), z)
        assert torch.allclose(grad, want, atol=1e-12)
    t = torch.tensor([3, 28, -1])
    top = z.detach().topk(4, 1).indices
    g = [torch.randn(3, dtype=torch.float64) for _ in range(3)] + [torch.randn(3, 4, dtype=torch.float64)]
    lp, lse, ent, _, _ = ref.logprobs64(z, t, 0, 0.7)
    total = (g[0] * lp).sum() + (g[1] * lse).sum() + (g[2] * ent).sum() \
        + (g[3] * torch.log_softmax(z / 0.7, 1).gather(1, top)).sum()
    want, = torch.autograd.grad(total, z)
    grad, _ = ref.backward64(z.detach(), t, 0.7, g[0], g[1], g[2], top, g[3])
    assert torch.allclose(grad, want, atol=1e-12)
