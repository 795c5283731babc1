"""The dropout module: where it draws no mask, and what it draws its masks from.  No GPU is used."""
import copy

import pytest
import torch
import torch.utils.checkpoint

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200 import autograd  # noqa: E402
from paper_2506_02939_b200.autograd import Dropout  # noqa: E402


@pytest.fixture
def drawn(monkeypatch):
    """(seed, offset) of every mask, instead of the mask."""
    seen = []
    monkeypatch.setattr(autograd, "dropout", lambda X, p, seed, offset=0, counter=None, residual=None: seen.append((seed, offset)) or X * 1.0)
    return seen


@pytest.mark.parametrize("module", [Dropout(0.5).eval(), Dropout(0.0)])
def test_the_residual_is_taken_in_the_inputs_type_and_shape(module):
    x, r = torch.randn(4, 8).bfloat16(), torch.randn(4, 8)
    y = module(x, r)
    assert y.dtype == torch.bfloat16 and torch.equal(y, x + r.bfloat16())
    y = module(r, x)
    assert y.dtype == torch.float32 and torch.equal(y, r + x.float())
    assert module(x) is x
    with pytest.raises(ValueError):
        module(x, r[:1])


def test_modules_are_independent_by_default(drawn):
    x = torch.ones(3)
    a, b = Dropout(0.5), Dropout(0.5)
    torch.manual_seed(1)
    for m in (a, b, a, b, copy.deepcopy(a)):
        m(x)
    assert len(set(drawn)) == 5 and all(0 <= s < 1 << 64 for s, _ in drawn)
    torch.manual_seed(1)
    again = Dropout(0.5)
    for _ in range(5):
        again(x)
    assert drawn[5:] == drawn[:5]
    a.eval()(x)                                              # draws nothing
    Dropout(0.0)(x)
    state = torch.get_rng_state()
    torch.manual_seed(1)
    for _ in range(5):
        torch.empty((), dtype=torch.int64).random_()
    assert len(drawn) == 10 and torch.equal(state, torch.get_rng_state())


def test_a_seed_numbers_the_calls(drawn):
    x = torch.ones(3)
    state = torch.get_rng_state()
    a, b = Dropout(0.5, seed=4), Dropout(0.5, seed=4)
    for m in (a, a, b, b):
        m(x)
    assert drawn[:2] == drawn[2:] == [(4, 1 << 32), (4, 2 << 32)] and torch.equal(state, torch.get_rng_state())


@pytest.mark.parametrize("reentrant", [False, True])
def test_checkpointing_draws_the_same_masks_again(drawn, reentrant):
    x = torch.ones(3, requires_grad=True)
    a, b = Dropout(0.5), Dropout(0.5)
    y = torch.utils.checkpoint.checkpoint(lambda t: b(a(t) * 2.0).exp(), x, use_reentrant=reentrant)
    torch.rand(5)                                            # something else draws in between
    y.sum().backward()
    assert len(drawn) == 4 and drawn[2:] == drawn[:2] and drawn[0] != drawn[1]


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_seeded_module_is_refused_in_a_backward_pass(drawn, reentrant):
    x = torch.ones(3, requires_grad=True)
    module = Dropout(0.5, seed=4)
    y = torch.utils.checkpoint.checkpoint(lambda t: module(t).exp(), x, use_reentrant=reentrant)
    with pytest.raises(RuntimeError, match="seed"):
        y.sum().backward()
    assert drawn == [(4, 1 << 32)] and module.calls == 1
    module(x).sum().backward()                               # outside it works on
    module.eval()                                            # and in evaluation mode anywhere
    torch.utils.checkpoint.checkpoint(lambda t: module(t).exp(), x, use_reentrant=reentrant).sum().backward()


def test_a_resumed_run_goes_on_with_the_masks(drawn, tmp_path):
    x = torch.ones(3)
    a = torch.nn.Sequential(Dropout(0.5, seed=4), Dropout(0.5))
    for _ in range(3):
        a(x)
    torch.save(a.state_dict(), tmp_path / "state.pt")
    b = torch.nn.Sequential(Dropout(0.5, seed=4), Dropout(0.5))
    b.load_state_dict(torch.load(tmp_path / "state.pt"))
    a[0](x), b[0](x)
    assert drawn[-1] == drawn[-2] == (4, 4 << 32)
    b.load_state_dict({})                                    # one that does not have the number
    assert b[0].calls == 4
    with pytest.raises(RuntimeError):
        b.load_state_dict({"2.weight": x})
