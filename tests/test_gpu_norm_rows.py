"""The norm's gradients where a block takes several rows: those that stay in
registers, and the longest, whose weight gradient is summed four rows at a time."""
import numpy as np
import pytest
import torch

from tests.logits_common import norm_backward_reference
from tests.train_common import check

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32

# 1,024 blocks to 8,192 columns, 256 beyond: two rows and more a block, the last trip not whole
SIZES = [(2500, 520), (1100, 1025), (2100, 2056), (1030, 4104), (2051, 8192), (530, 8200), (600, 16384), (259, 16392), (1300, 16500),
         (1027, 20001), (600, 32776), (515, 65536)]


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,D", SIZES)
def test_backward_of_many_rows(dv, N, D, dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(N + D)
    make = lambda n, scale: (torch.randn((n, D), generator=g, device=DEV) * scale).to(dtype)  # noqa: E731
    h, grad, gt, w = make(N, 2.0), make(N, 1.0), make(N, 0.5), make(1, 1.0)[0]
    rstd = (1.0 / torch.sqrt((h.double() ** 2).mean(1) + 1e-5)).float()
    for grad_total in (gt, None):
        gx, gw = dv.rms_norm_backward(grad, h, w, rstd, grad_total=grad_total)
        # (the reference's arrays in 64 bits: on the device, rows at a time for grad_x)
        *_, dw, dw_tol = norm_backward_reference(grad, h, w, rstd, grad_total)
        check(gw, dw.cpu(), dw_tol.cpu(), "grad_weight")
        for i in range(0, N, 512):
            r = slice(i, min(N, i + 512))
            dx, dx_tol, _, _ = norm_backward_reference(grad[r], h[r], w, rstd[r], None if grad_total is None else grad_total[r])
            off = (gx[r].double() - dx).abs()
            assert bool((off <= dx_tol).all()), f"grad_x of rows {i} on: {float((off - dx_tol).max())} beyond its bound"
        only_x, _ = dv.rms_norm_backward(grad, h, w, rstd, grad_total=grad_total, want_weight=False)
        _, only_w = dv.rms_norm_backward(grad, h, w, rstd, grad_total=grad_total, want_x=False)
        assert torch.equal(only_x, gx) and torch.equal(only_w, gw)
