"""The dropout module's masks and types."""
import pytest
import torch
import torch.utils.checkpoint

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200.autograd import Dropout  # noqa: E402

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def normal(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("types", [(BF16, F32), (F32, BF16)])
def test_a_residual_of_another_type_in_every_mode(types):
    x, r = normal((9, 40), types[0], 1).requires_grad_(), normal((9, 40), types[1], 2).requires_grad_()
    module = Dropout(0.5, seed=3)
    train = module(x, r)
    evaluated, none = module.eval()(x, r), Dropout(0.0)(x, r)
    assert torch.equal(evaluated, x + r.to(types[0])) and torch.equal(none, evaluated)
    for y in (train, evaluated, none):
        assert y.dtype == types[0]
        x.grad = r.grad = None
        y.backward(torch.ones_like(y))
        assert x.grad.dtype == types[0] and r.grad.dtype == types[1] and (r.grad == 1).all()
    same = Dropout(0.5, seed=3)(x, r.to(types[0]))
    assert torch.equal(train, same)


@pytest.mark.parametrize("reentrant", [False, True])
def test_two_layers_under_checkpointing(reentrant):
    """The masks of two modules differ, and the gradient has the ones that the loss had."""
    x = normal((64, 128), F32, 4).requires_grad_()
    a, b = Dropout(0.5), Dropout(0.5)
    seen = []

    def layers(t):
        one = a(t)
        two = b(torch.ones_like(t))
        seen.append((one.detach() != 0, two.detach() != 0))
        return one * two

    y = torch.utils.checkpoint.checkpoint(layers, x, use_reentrant=reentrant)
    torch.rand(3)
    y.sum().backward()
    (m, n), again = seen
    assert torch.equal(m, again[0]) and torch.equal(n, again[1]) and not torch.equal(m, n)
    assert torch.equal(x.grad, torch.where(m & n, 4.0, 0.0))


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_seeded_module_is_refused_in_a_backward_pass(reentrant):
    x = normal((8, 16), F32, 5).requires_grad_()
    module = Dropout(0.5, seed=4)
    y = torch.utils.checkpoint.checkpoint(lambda t: module(t).exp(), x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="seed"):
        y.sum().backward()
    again = Dropout(0.5, seed=4)
    again(x)
    assert torch.equal(module(x), again(x))
