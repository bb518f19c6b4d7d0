"""A teacher's token whose logit is near the type's lowest value, at inverse
temperatures above 1: a large loss, but a finite one where it is finite."""
import numpy as np
import pytest
import torch

from tests.test_gpu_distill import make, run
from tests.train_common import check, distill_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(3, 700), (2, 90001), (300, 1200)])
@pytest.mark.parametrize("c", [1.0, 1.25, 4.0])
def test_listed_token_of_the_lowest_value(dv, dtype, N, V, c):
    z, ids, top, _, _, mask, g = make(13, N, V, 6, dtype, 0)
    ids[:] = torch.from_numpy(np.arange(6, dtype=np.int32) * 3)
    z[:, 0] = torch.finfo(dtype).min
    top[:, 1:] = 8.0
    top[:, 0] = 8.0 - 4.5 / c  # a probability of about 0.0022
    ref = distill_reference(z, ids, top, c, mask, g)
    assert bool((ref["loss"] > 1e35).all() & (ref["loss"] < 3e38).all())
    alone, loss, grad = run(dv, z, ids, top, c, None, None, g)
    check(loss, ref["loss"], ref["loss_tol"], "loss")
    check(alone, ref["loss"], ref["loss_tol"], "loss alone")
    check(grad, ref["grad"], ref["grad_tol"], "grad")
