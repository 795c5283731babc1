"""The dropout module where it draws no mask; no GPU is used."""
import pytest
import torch

from paper_2506_02939_b200 import build as pamm_build

pamm_build.build()
from paper_2506_02939_b200.autograd import Dropout  # noqa: E402


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
