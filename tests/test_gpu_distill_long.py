"""Distillation of rows so long that few are under way at once: a block a compute
unit, or two."""
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


@pytest.mark.parametrize("N,V,dtype,masked", [
    (161, 150001, torch.bfloat16, True), (165, 230003, torch.bfloat16, True), (160, 256000, torch.bfloat16, False),
    (162, 75001, torch.float32, False), (163, 120007, torch.float32, True),
])
def test_matches_the_64_bit_form(dv, N, V, dtype, masked):
    print(f"distill long N={N} V={V} {dtype} masked={masked}", flush=True)
    z, ids, top, may, states, mask, g = make(N, N, V, 9, dtype, 4 if masked else 0)
    for c, pad, in_place in ((1.0, 0, False), (0.5, 3, True)):
        ref = distill_reference(z, ids, top, c, mask, g)
        alone, loss, grad = run(dv, z, ids, top, c, may, states, g, pad, in_place)
        check(loss, ref["loss"], ref["loss_tol"], "loss")
        check(alone, ref["loss"], ref["loss_tol"], "loss alone")
        check(grad, ref["grad"], ref["grad_tol"], "grad")
