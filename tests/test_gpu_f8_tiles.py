"""The 256 x 256 tiles of 8-bit products, which large training steps run: several
blocks of k, b by tiles and by rows, sums of parts, rows far apart."""
import numpy as np
import pytest
import torch

from tests.logits_common import B, product_reference, quantize
from tests.train_common import check

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def whole_numbers(rng, M, N, K, tile):
    """Operands whose products nothing cuts: whole numbers to 15 of either sign, products below 2^8, under scales of
    1/2, 1 and 2: every sum is a multiple of 2^-2 and, of terms of random sign, far below 2^22 (some
    2^8 sqrt(K) 2), so exact in fp32."""
    small = torch.arange(16).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    one = lambda n: torch.from_numpy(small[rng.integers(0, 16, (n, K))] | (rng.integers(0, 2, (n, K)) << 7).astype(np.uint8))  # noqa: E731
    power = lambda *s: torch.from_numpy(2.0 ** rng.integers(-1, 2, s)).float()  # noqa: E731
    kb = K // B
    sb = power(kb, N) if tile == 1 else power((N + B - 1) // B, kb)
    return one(M).view(torch.float8_e4m3fn), power(kb, M), one(N).view(torch.float8_e4m3fn), sb


def exact_rows(a, sa, b, sb, tile, rows):
    """The product's rows in float64, on the device (a float64 product is not batched)."""
    va = a[rows].to(DEV).float().double() * sa[:, rows].t().double().repeat_interleave(B, 1).to(DEV)
    s = sb.double().to(DEV)
    s = s.t() if tile == 1 else s.repeat_interleave(B, 0)[:b.shape[0]]
    return va @ (b.to(DEV).float().double() * s.repeat_interleave(B, 1)).t()


# none of them in parts; the last has 44 blocks of k
SHAPES = [(3000, 3100, 128), (3000, 3100, 256), (3000, 3100, 384), (4097, 4100, 512), (2817, 4096, 1152), (4000, 4096, 5632)]


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_whole_numbers_to_the_last_bit(dv, M, N, K, tile):
    rng = np.random.default_rng(M + K + tile)
    a, sa, b, sb = whole_numbers(rng, M, N, K, tile)
    wide = torch.full((M, N + 5), 3.0, dtype=BF, device=DEV)
    dv.product_f8(a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV), tile=tile, out=wide[:, 2:N + 2])
    assert (wide[:, :2] == 3).all() and (wide[:, N + 2:] == 3).all()
    for r in range(0, M, 1024):
        rows = slice(r, min(M, r + 1024))
        assert torch.equal(wide[rows, 2:N + 2], exact_rows(a, sa, b, sb, tile, rows).to(BF))


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K", [(1024, 4096, 32000), (1000, 4090, 16128)])
def test_whole_numbers_in_parts(dv, M, N, K, tile):
    """A long sum in parts of 256 x 256 tiles, joined."""
    rng = np.random.default_rng(K)
    a, sa, b, sb = whole_numbers(rng, M, N, K, tile)
    need = dv.product_f8_workspace_bytes(M, N, K)
    assert need > 0
    ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device=DEV)
    out = dv.product_f8(a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV), tile=tile, workspace=ws[:need])
    assert (ws[need:] == 0xFF).all()
    assert torch.equal(out, exact_rows(a, sa, b, sb, tile, slice(0, M)).to(BF))


@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K", [(3000, 3100, 384), (2817, 4096, 1152)])
def test_normal_values(dv, M, N, K, tile):
    """Sampled rows within their bound, and the error of all of them in the mean of squares
    within the result's rounding (2^-9 of it at most)."""
    rng = np.random.default_rng(K)
    a, sa = quantize(torch.from_numpy(rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, 1)))).float(), 1)
    b, sb = quantize(torch.from_numpy(rng.normal(size=(N, K)) * np.exp(rng.normal(size=(N, 1)))).float(), tile)
    out = dv.product_f8(a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV), tile=tile)
    off = out.double() - exact_rows(a, sa, b, sb, tile, slice(0, M))
    assert float((off.square().sum() / out.double().square().sum()).sqrt()) < 2.0 ** -9
    rows = torch.from_numpy(np.sort(rng.choice(M, 300, replace=False)))
    want, tol = product_reference(a[rows], sa[:, rows], b, sb, tile, BF)
    check(out[rows.to(DEV)], want, tol, "sampled rows")


def test_rows_far_apart(dv):
    """The widest row strides under 256-row tiles: 255 rows lie 2^30 bytes apart, of either operand."""
    rng = np.random.default_rng(7)
    M, N, K = 3000, 3100, 256
    a, sa, b, sb = whole_numbers(rng, M, N, K, 128)
    a, sa, b, sb = (t.to(DEV) for t in (a, sa, b, sb))
    want = dv.product_f8(a, sa, b, sb)

    def far(t):
        wide = torch.empty((t.shape[0] - 1) * (1 << 22) + K, dtype=torch.uint8, device=DEV)
        torch.as_strided(wide, t.shape, (1 << 22, 1)).copy_(t.view(torch.uint8))
        return torch.as_strided(wide.view(dv.F8), t.shape, (1 << 22, 1))

    assert torch.equal(dv.product_f8(far(a), sa, b, sb), want)
    torch.cuda.empty_cache()
    assert torch.equal(dv.product_f8(a, sa, far(b), sb), want)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("M,N,K", [(1, 500, 1152), (16, 130, 384), (31, 1000, 2176), (64, 257, 640), (65, 500, 128), (129, 300, 256),
                                   (250, 700, 1664), (257, 513, 384), (300, 260, 6016), (520, 1030, 512), (1300, 2100, 640)])
def test_whole_numbers_of_every_kernel(dv, M, N, K, tile, dtype):
    """The streamed kernels, the exact and the 8-bit tiles of 128, in parts and not: nothing is lost."""
    rng = np.random.default_rng(M * 3 + K)
    a, sa, b, sb = whole_numbers(rng, M, N, K, tile)
    out = dv.product_f8(a.to(DEV), sa.to(DEV), b.to(DEV), sb.to(DEV), tile=tile, dtype=dtype)
    assert torch.equal(out, exact_rows(a, sa, b, sb, tile, slice(0, M)).to(dtype))
