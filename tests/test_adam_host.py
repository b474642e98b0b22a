"""Host-only checks of the AdamW plan: what is refused before CUDA is touched, and the tests' own reference."""
import ctypes

import pytest
import torch

import adam_reference as ref


@pytest.fixture(scope="module")
def qn():
    from paper_1709_05069_b200 import build as qn_build
    from paper_1709_05069_b200 import qn as mod

    qn_build.build()
    mod.lib()
    return mod


def test_bad_plans_are_refused_before_cuda(qn):
    L, bad, out = qn.lib(), qn.QN_ERR_INVALID, ctypes.c_void_p(1)
    host = (ctypes.c_char * 4096)()
    p = ctypes.addressof(host)
    table = (qn._AdamTensor * 1)(qn._AdamTensor(8, p, p + 64, None, p + 128, p + 192, None, None, 0.0, 1.0))
    at = ctypes.addressof(table)
    for args in ((-1, at, 0, 0, 0), (1, None, 0, 0, 0), (1, at, 5, 0, 0), (1, at, 0, 7, 0), (1, at, 0, 0, 2), (1, at, 0, 0, 0)):
        # the last one has nothing wrong but that its memory is the host's
        assert L.qn_adam_create(*args, ctypes.byref(out)) == bad and not out.value
    assert L.qn_adam_create(1, at, 0, 0, 0, None) == bad
    table[0].numel = -1
    assert L.qn_adam_create(1, at, 0, 0, 0, ctypes.byref(out)) == bad
    assert L.qn_adam_destroy(None) == bad and L.qn_adam_norm(None, p, None) == bad and L.qn_adam_grads(None, p, None) == bad
    assert L.qn_adam_state(None, 0, p, p, None) == bad and L.qn_adam_places(None) == 0
    assert L.qn_adam_step(None, p, 1e-3, None, 0.9, 0.999, 1e-8, None, 0.0, 1.0, 0, 0, None) == bad


def test_binding_refuses_host_tensors(qn):
    x = torch.zeros(8)
    with pytest.raises(ValueError, match="CUDA tensors"):
        qn.qn_adam_create([x], [x.clone()], [x.clone()], [x.clone()])


@pytest.mark.parametrize("fraction", [3, 4])
def test_codes_of_the_reference_are_the_format(fraction):
    """Every code's value is coded as itself whatever the chance, and a value between two becomes the upper one as often as
    it is far from the lower."""
    codes = torch.arange(256)[: 256 if fraction == 4 else 127].to(torch.uint8)
    codes = codes[codes <= (0x70 if fraction == 3 else 0xF0 - 16)]
    if fraction == 3:
        e4m3 = codes.view(torch.float8_e4m3fn).double()
        assert torch.equal(ref.decode(codes, torch.full((4,), 127, dtype=torch.uint8), 3), e4m3)
    scale = torch.full(((codes.numel() + 31) // 32,), 100, dtype=torch.uint8)
    values = ref.decode(codes, scale, fraction)
    for chance in (0, 1 << 15, 65535):
        again = ref.encode(values, scale, torch.full(codes.shape, chance), fraction)
        assert torch.equal(again, codes)
    middle = (values[:-1] * 3 + values[1:]) / 4
    up = sum((ref.encode(middle, scale, torch.full(middle.shape, c), fraction) == codes[1:]).double() for c in range(0, 65536, 512)) / 128
    low = 1 if fraction == 4 else 0  # nothing but 0 has the root's code 0
    assert torch.allclose(up[low:], torch.full_like(up[low:], 0.25), atol=1e-9)


def test_words_are_even():
    w = ref.words(ref.step_key(11, 5), torch.arange(1 << 16))
    for x in ((w >> 16), (w & 65535)):
        # the mean of 2^16 numbers even on [0, 1): a standard error of 1 / sqrt(12 * 2^16); five are allowed
        assert abs(float((x.double() / 65536).mean()) - 0.5) < 5 / (12 * 65536) ** 0.5
    assert len(set(ref.step_key(s, t) for s in (0, 1, 1 << 32) for t in (0, 1, 2, 1 << 32))) == 12
