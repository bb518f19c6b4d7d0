"""Arrays of more than 2^31 elements and 2^32 bytes through the operators from the
last layer to the logits: their ends equal the same calls on the ends alone (a
product's, whose parts a small call adds up in another order, its 64-bit form)."""
import pytest
import torch

from tests.logits_common import product_reference
from tests.train_common import check

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF = torch.bfloat16


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def rows(n, d, seed):
    """[n][d] bf16: a thousand normal rows, again and again, each time a little larger."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    some = torch.randn((1000, d), generator=g, device=DEV)
    out = torch.empty((n, d), dtype=BF, device=DEV)
    for k, i in enumerate(range(0, n, 1000)):
        out[i:i + 1000] = (some[:n - i] * (1 + k * 1e-3)).to(BF)
    return out


def same(a, b):
    a, b = (t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t for t in (a, b))
    return torch.equal(a, b)


def test_norm(dv):
    N, D = 540_000, 4104
    assert N * D > 1 << 31
    x, w = rows(N, D, 1), torch.ones(D, dtype=BF, device=DEV)
    out, total, rstd = dv.rms_norm(x, w, residual=x, want_rstd=True)
    for cut in (slice(0, 9), slice(N - 9, N)):
        o, t, r = dv.rms_norm(x[cut], w, residual=x[cut], want_rstd=True)
        assert same(out[cut], o) and same(total[cut], t) and same(rstd[cut], r)
    del out
    gx, _ = dv.rms_norm_backward(x, total, w, rstd, want_weight=False)
    for cut in (slice(0, 9), slice(N - 9, N)):
        assert same(gx[cut], dv.rms_norm_backward(x[cut], total[cut], w, rstd[cut], want_weight=False)[0])
    del gx, total
    q, s, _ = dv.rms_norm_f8(x, w)
    q2, s2, _ = dv.rms_norm_f8(x[N - 9:], w)
    assert same(q[N - 9:], q2) and same(s[:, N - 9:], s2)


@pytest.mark.parametrize("tile", [1, 128])
def test_quantize(dv, tile):
    N, K = 66_000, 33_000
    assert N * K > 1 << 31
    x = rows(N, K, 2)
    q, s, tq, ts = dv.quantize_f8(x, tile=tile, want_columns=True)
    n0 = N // 128 * 128 - 256                       # whole blocks of rows before the end
    q2, s2, tq2, ts2 = dv.quantize_f8(x[n0:], tile=tile, want_columns=True)
    assert same(q[n0:], q2) and same(tq[:, n0:], tq2)
    if tile == 1:
        assert same(s[:, n0:], s2) and same(ts[n0 // 128:], ts2)
    else:
        assert same(s[n0 // 128:], s2) and same(ts[:, n0 // 128:], ts2)


@pytest.mark.parametrize("M,N,K", [(40_000, 60_000, 128), (3, 1 << 21, 2176), (70, 1 << 20, 4224)])
def test_product(dv, M, N, K):
    """More than 2^31 results, or 2^32 bytes of b (streamed, and in tiles)."""
    assert M * N > 1 << 31 or N * K > 1 << 32
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    a = dv.quantize_f8(torch.randn((M, K), generator=g, device=DEV))[:2]
    b = torch.empty((N, K), dtype=dv.F8, device=DEV)
    some = torch.randint(0, 0x70, (4096, K), generator=g, device=DEV, dtype=torch.uint8)
    for i in range(0, N, 4096):
        b.view(torch.uint8)[i:i + 4096] = some[:N - i]
    sb = torch.rand(((N + 127) // 128, K // 128), generator=g, device=DEV) + 0.5
    out = dv.product_f8(*a, b, sb)
    n0 = N // 128 * 128 - 512                       # whole tiles before the end
    rows_ = slice(M - 300, M) if M > 300 else slice(0, M)
    want, tol = product_reference(a[0][rows_].cpu(), a[1][:, rows_].cpu(), b[n0:].cpu(), sb[n0 // 128:].cpu(), 128, BF)
    check(out[rows_, n0:], want, tol, "the end of the product")


def test_adjust(dv):
    B, V = 17_000, 128_256
    assert B * V > 1 << 31
    z = rows(B, V, 4)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    hist = torch.randint(0, V, (B, 20), generator=g, device=DEV, dtype=torch.int32)
    lengths = torch.full((B,), 20, dtype=torch.int32, device=DEV)
    rep = torch.full((B,), 1.25, device=DEV)
    out = dv.adjust_logits(z, hist, lengths, repetition=rep)
    part = dv.adjust_logits(z[B - 5:], hist[B - 5:], lengths[B - 5:], repetition=rep[B - 5:])
    assert same(out[B - 5:], part) and not same(part, z[B - 5:])
    dv.adjust_logits(z, hist, lengths, repetition=rep, out=z)
    assert torch.equal(z[B - 5:], part)
