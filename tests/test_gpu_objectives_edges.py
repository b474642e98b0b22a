"""qn_policy: calls that its documentation does not allow."""
import pytest
import torch

from test_gpu_objectives import BF16, F32, qn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_policy_gradient_over_its_other_inputs_is_refused(qn, dtype):  # noqa: F811
    """The gradient of one row would take the place of what another row still has to read."""
    rows, vocab = 6, 40
    z = torch.randn(rows, vocab, device="cuda").to(dtype)
    arena = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    size = z.element_size()

    def side(at, kind):
        return arena[at:at + rows * (8 if kind is torch.int64 else 4)].view(kind)

    d = arena[64:64 + rows * vocab * size].view(dtype).view(rows, vocab)
    end = 64 + rows * vocab * size
    for name in ("tokens", "old_logprob", "ref_logprob", "advantage", "weight"):
        kind = torch.int64 if name == "tokens" else F32
        each = 8 if kind is torch.int64 else 4
        for at, over in ((64 - rows * each, False), (72 - rows * each, True), (256, True), (end - 8, True), (end, False)):
            args = dict(logits=z, tokens=torch.zeros(rows, dtype=torch.int64, device="cuda"), kl=0.1, loss=torch.full((rows,), 9.0, device="cuda"),
                        **{x: torch.ones(rows, device="cuda") for x in ("old_logprob", "ref_logprob", "advantage", "weight")}, dlogits=d)
            if at < 0:
                continue
            args[name] = side(at, kind)
            arena.zero_()
            if name == "weight":
                args[name].fill_(1.0)
            if over:
                with pytest.raises(qn.QNError):
                    qn.qn_policy(**args)
                assert bool((args["loss"] == 9.0).all())
            else:
                qn.qn_policy(**args)
                assert bool(torch.isfinite(d).all()) and bool(d.any()) and not bool((args["loss"] == 9.0).any())


@pytest.mark.parametrize("name", ["tokens", "old_logprob", "ref_logprob", "advantage", "weight"])
def test_policy_inputs_between_the_rows_of_its_gradient(qn, name):  # noqa: F811
    """What lies wholly between two rows of the gradient is as far from it as anything else; what reaches into a row is not."""
    rows, vocab, stride = 3, 8, 24
    gen = torch.Generator(device="cuda").manual_seed(1)
    z = torch.randn(rows, vocab, generator=gen, device="cuda")
    given = {x: torch.randn(rows, generator=gen, device="cuda") for x in ("old_logprob", "ref_logprob", "advantage", "weight")}
    given["tokens"] = torch.tensor([1, 7, 0], device="cuda")
    want_loss, want = torch.empty(rows, device="cuda"), torch.empty_like(z)
    qn.qn_policy(z, loss=want_loss, dlogits=want, kl=0.1, **given)
    each = given[name].element_size() // 4 * rows
    for row in range(rows - 1):
        for at, apart in ((stride * row + vocab, True), (stride * (row + 1) - each, True), (stride * row + vocab - 2, False),
                          (stride * (row + 1) - each + 2, False)):
            store = torch.full((rows * stride,), 5.0, device="cuda")
            d, args, loss = store.as_strided((rows, vocab), (stride, 1)), dict(given), torch.full((rows,), 9.0, device="cuda")
            args[name] = store[at:at + each].view(given[name].dtype)
            args[name].copy_(given[name])
            if apart:
                qn.qn_policy(z, loss=loss, dlogits=d, kl=0.1, **args)
                assert torch.equal(loss, want_loss) and torch.equal(d, want) and torch.equal(args[name], given[name])
            else:
                with pytest.raises(qn.QNError):
                    qn.qn_policy(z, loss=loss, dlogits=d, kl=0.1, **args)
