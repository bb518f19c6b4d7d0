"""Products of 8-bit operands whose two scales together leave the range of fp32,
where the results do not: each kernel, b by tiles and by rows."""
import math

import numpy as np
import pytest
import torch

from tests.logits_common import B, U, own_rounding, values
from tests.train_common import check

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32

# few rows (three kernels), exact tiles, 8-bit tiles of 128, of 256 and several blocks of k
SIZES = [(5, 300, 256, F32), (24, 200, 640, F32), (40, 300, 256, BF), (150, 300, 384, F32), (150, 300, 384, BF),
         (300, 260, 256, BF), (3000, 3100, 384, BF)]


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def operands(rng, M, N, K, tile, least=0x70):
    """Positive e4m3 values (from 128 on) and scales of 1 to 2."""
    one = lambda n: torch.from_numpy(rng.integers(least, 0x7F, (n, K)).astype(np.uint8))  # noqa: E731
    scales = lambda *s: torch.from_numpy(1 + rng.random(s)).float()  # noqa: E731
    sb = scales(K // B, N) if tile == 1 else scales((N + B - 1) // B, K // B)
    return one(M), scales(K // B, M), one(N), sb


def product(dv, a, sa, b, sb, tile, dtype):
    f8 = lambda t: t.to(DEV).view(dv.F8)  # noqa: E731
    return dv.product_f8(f8(a), sa.to(DEV), f8(b), sb.to(DEV), tile=tile, dtype=dtype)


def reference(a, sa, b, sb, tile, dtype):
    """Terms of one sign, so that the sums' magnitudes are the results: a relative bound alone (the sum in the
    instruction, the scales, a sum of blocks, the cut of the 8-bit instruction), and the steps of
    subnormal results, one for each block of k and 2^-133 of bf16's."""
    va = values(a.view(torch.float8_e4m3fn), sa, 1)
    vb = values(b.view(torch.float8_e4m3fn), sb, tile)
    y = va @ vb.t()
    kb = a.shape[1] // B
    rel = (2 * B + kb + 4) * U + own_rounding(dtype) + (7 * 2.0 ** -13 if dtype == BF and a.shape[0] > 256 else 0)
    return y, rel * 1.01 * y.abs() + (kb + 2) * 2.0 ** -149 + (2.0 ** -133 if dtype == BF else 0)


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K,dtype", SIZES, ids=lambda v: str(v).replace("torch.", ""))
@pytest.mark.parametrize("ea,eb", [(-72, -72), (-20, -125), (-125, -20), (-108, -30), (115, -100), (-100, 115), (60, 38), (-109, 119)])
def test_scales_of_all_sizes(dv, ea, eb, M, N, K, dtype, tile):
    """2^ea and 2^eb: together subnormal, or one of them so large that it leaves no room for a block's sum."""
    a, sa, b, sb = operands(np.random.default_rng(M + K), M, N, K, tile)
    sa, sb = sa * 2.0 ** ea, sb * 2.0 ** eb
    want, tol = reference(a, sa, b, sb, tile, dtype)
    check(product(dv, a, sa, b, sb, tile, dtype), want, tol, f"scales 2^{ea}, 2^{eb}")


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K,dtype", SIZES, ids=lambda v: str(v).replace("torch.", ""))
def test_a_block_of_zeros_beside_large_scales(dv, M, N, K, dtype, tile):
    """A block's products all zero under scales whose product is past fp32's largest add nothing."""
    a, sa, b, sb = operands(np.random.default_rng(M + K + 1), M, N, K, tile)
    a[:, B:B + 64] = 0
    b[:, B + 64:2 * B] = 0
    want, tol = reference(a, sa, b, sb, tile, dtype)
    sa[1] *= 2.0 ** 100
    if tile == 1:
        sb[1] *= 2.0 ** 100
    else:
        sb[:, 1] *= 2.0 ** 100
    check(product(dv, a, sa, b, sb, tile, dtype), want, tol, "beside zeros")


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K,dtype", SIZES, ids=lambda v: str(v).replace("torch.", ""))
def test_results_past_the_largest(dv, M, N, K, dtype, tile):
    """Infinities of the right sign, beside finite rows; scales of zero, infinity and NaN as they multiply."""
    a, sa, b, sb = operands(np.random.default_rng(M + K + 2), M, N, K, tile)
    a[1] |= 0x80
    sa[:, :2] *= 2.0 ** 60
    sb *= 2.0 ** 55
    sa[:, 2] = 0
    sa[:, 3] = math.inf
    sa[0, 4] = math.nan
    out = product(dv, a, sa, b, sb, tile, dtype).cpu()
    assert (out[0] == math.inf).all() and (out[1] == -math.inf).all() and (out[2] == 0).all()
    assert (out[3] == math.inf).all() and torch.isnan(out[4]).all()
    if M > 5:
        want, tol = reference(a[5:], sa[:, 5:], b, sb, tile, dtype)
        check(out[5:], want, tol, "beside infinities")


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_quantized_far_from_one(dv, dtype, tile):
    """From arrays to logits: values near 2^-75 on both sides, and 2^110 against 2^-100."""
    rng = np.random.default_rng(8)
    x, w = (torch.from_numpy(rng.random((n, 256)) + 0.5).float() for n in (70, 150))
    for ex, ew in ((-75, -52), (110, -100), (-100, 110)):
        xs, ws = (x * 2.0 ** ex).to(DEV), (w * 2.0 ** ew).to(DEV)
        q, s = dv.quantize_f8(xs)[:2]
        wq, wsc = dv.quantize_f8(ws, tile=tile)[:2]
        want, tol = reference(q.cpu().view(torch.uint8), s.cpu(), wq.cpu().view(torch.uint8), wsc.cpu(), tile, dtype)
        check(dv.product_f8(q, s, wq, wsc, tile=tile, dtype=dtype), want, tol, "quantized")
