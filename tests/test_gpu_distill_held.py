"""Distillation of logits larger than the caches, whose rows the kernels hold in
registers: each block shape against the 64-bit form, with masks, strides,
in-place gradients, and rows of lowest values, -infinity and NaN among them."""
import math

import pytest
import torch

from tests.test_gpu_distill import make, run
from tests.train_common import check, distill_reference

pytestmark = pytest.mark.gpu

BF, F = torch.bfloat16, torch.float32
# logits of 32 MB and more, tokens around the block shapes' limits and between
SIZES = [(8500, 2001, BF), (4300, 4103, BF), (2200, 8191, BF), (1050, 16391, BF), (560, 32767, BF), (530, 33001, BF),
         (1000, 60001, BF), (8500, 1001, F), (4200, 2051, F), (1100, 8191, F), (500, 16383, F), (505, 32767, F),
         (250, 50257, F)]


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


@pytest.mark.parametrize("N,V,dtype", SIZES)
@pytest.mark.parametrize("masked", [False, True])
def test_matches_the_64_bit_form(dv, N, V, dtype, masked):
    print(f"distill held N={N} V={V} {dtype} masked={masked}", flush=True)
    K = 21
    z, ids, top, may, states, mask, g = make(N + V, N, V, K, dtype, 4 if masked else 0)
    lowest = torch.finfo(dtype).min
    z[3] = lowest                     # uniform
    z[4, : V // 2] = lowest           # these never count
    clean = z.clone()
    if masked:
        z[5:9][~mask[5:9]] = float("nan")
        z[9:12][~mask[9:12]] = math.inf
    for c, pad, in_place in ((1.25, 0, False), (0.5, 3, True)):
        ref = distill_reference(clean, ids, top, c, mask, g)
        _, loss, grad = run(dv, z, ids, top, c, may, states, g, pad, in_place)
        want = ref["loss"].clone()
        want[want > torch.finfo(torch.float32).max] = math.inf  # a listed lowest value may pass the loss's range
        check(loss, want, ref["loss_tol"], "loss")
        check(grad, ref["grad"], ref["grad_tol"], "grad")


@pytest.mark.parametrize("N,V,dtype", [(2200, 8191, BF), (1000, 60001, BF), (250, 50257, F)])
def test_rows_without_a_softmax(dv, N, V, dtype):
    z, ids, top, _, _, mask, g = make(7, N, V, 5, dtype, 0)
    empty, nan_first, nan_last = 2, 6, N - 1
    z[empty] = -math.inf
    z[nan_first, 0] = float("nan")
    z[nan_last, V - 1] = float("nan")
    _, loss, grad = run(dv, z, ids, top, 1.0, None, None, g)
    assert float(loss[empty]) == 0.0 and not grad[empty].any()
    assert bool(torch.isnan(loss[[nan_first, nan_last]]).all())
    keep = [0, 1, 3, 4, 5, 7, N - 2]
    ref = distill_reference(z[keep], ids[keep], top[keep], 1.0, mask[keep], g[keep])
    check(loss[keep], ref["loss"], ref["loss_tol"], "loss")
    check(grad[keep], ref["grad"], ref["grad_tol"], "grad")


def test_same_bits_each_time(dv):
    z, ids, top, may, states, mask, g = make(29, 1050, 16391, 9, BF, 3)
    a = run(dv, z, ids, top, 1.0, may, states, g)
    b = run(dv, z, ids, top, 1.0, may, states, g, in_place=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
