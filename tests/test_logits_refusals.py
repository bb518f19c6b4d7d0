"""Calls from the last layer to the logits that are refused (no GPU needed)."""
import pytest
import torch

import paper_2403_06988_amd as dv
from paper_2403_06988_amd import autograd as dva


@pytest.mark.parametrize("x,w", [((4, 100), (30, 120)), ((4, 100), (30, 128)), ((4, 128), (30, 100)), ((4, 256), (30, 128)),
                                 ((100,), (30, 100)), ((4, 100), (100,))])
def test_linear_f8_refuses_other_depths(x, w):
    """Operands are padded to whole blocks of 128: rows of 100 and 120 would both be 128 long."""
    with pytest.raises(ValueError, match="weight must be"):
        dva.linear_f8(torch.zeros(x), torch.zeros(w))
