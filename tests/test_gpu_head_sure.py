"""Losses of rows that are sure of their target: small, and as exact as their logits allow."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(1, 100), (3, 5000), (200, 3001), (2000, 6000)])
def test_small_losses(dv, N, V, dtype):
    """Logits that are whole numbers times 2^-3, exact in any order: the target's is the
    largest, the others lie 4 to 24 below it.  The loss ln(1 + s) of s = sum of exp(z - z_t) <=
    1: each exponential is off by its argument (a product of at most 24 log2(e) < 35, rounded:
    35 U ln 2 < 25 U) and 2 U, their sum by 8 U (16 of a tile's values a lane, tiles in pairs
    or 16 a lane: at most 64 roundings of partial sums of one sign, 64 U), the rescaling from
    tile to tile and to the target by 27 U each; log1p by 4 U."""
    g = torch.Generator().manual_seed(N + V)
    D = 64
    x = torch.zeros((N, D))
    x[:, 0], x[:, 1] = 1.0, 8.0
    w = torch.zeros((V, D))
    w[:, 0] = -torch.randint(5 * 8, 24 * 8, (V,), generator=g) / 8.0
    w[V // 3, 0] = 0.0
    few = torch.randperm(V, generator=g)[: V // 2]
    w[few, 0] = -20.0  # keeps s below 1
    w[V // 3, 0] = 0.0
    big = w[:, 0] > -12.0
    big[V // 3] = False
    w[big, 0] -= 8.0
    w[:, 1] = torch.full((V,), 1.5)  # all logits 12 higher: the loss does not know
    t = torch.full((N,), V // 3, dtype=torch.int32)
    loss, lse = dv.head_loss(x.to(dtype).to(DEV), w.to(dtype).to(DEV), t.to(DEV))
    wz = w.to(dtype).double()[:, 0]
    rest = torch.exp(wz[torch.arange(V) != V // 3] - wz[V // 3]).sum()
    assert 0 < rest < 1
    want = float(torch.log1p(rest))
    tol = (25 + 2 + 64 + 2 * 27 + 4 + 8) * 2.0 ** -24 * want
    assert bool(((loss.cpu().double() - want).abs() <= tol).all())
    assert bool(((lse.cpu().double() - (want + 12.0)).abs() <= 2.0 ** -20 + tol).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_only_allowed_token(dv, dtype):
    """Nothing but the target is allowed: the loss is 0, lse the target's logit; the
    row's gradient is 0."""
    N, D, V = 70, 64, 300
    g = torch.Generator().manual_seed(3)
    x, w = torch.randn((N, D), generator=g).to(dtype), torch.randn((V, D), generator=g).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, dtype=torch.int32)
    bits = torch.zeros((N, (V + 31) // 32), dtype=torch.int64)
    bits[torch.arange(N), t.long() // 32] = 1 << (t.long() % 32)
    allow = torch.where(bits >= 1 << 31, bits - (1 << 32), bits).int().to(DEV)
    states = torch.arange(N, dtype=torch.int32, device=DEV)
    args = (x.to(DEV), w.to(DEV), t.to(DEV))
    loss, lse = dv.head_loss(*args, allow=allow, states=states)
    z = (x.double() * w[t.long()].double()).sum(1)
    assert not loss.any()
    assert bool(((lse.cpu().double() - z).abs() <= 1e-5 * (1 + z.abs())).all())
    other = t.clone()
    other[:] = (t + 1) % V  # not allowed: no part, the same lse
    loss2, lse2 = dv.head_loss(args[0], args[1], other.to(DEV), allow=allow, states=states)
    assert not loss2.any() and torch.equal(lse, lse2)
    gx, gw = dv.head_loss_backward(*args, lse, torch.ones(N, device=DEV), allow=allow, states=states)
    assert math.isclose(float(gx.float().abs().max()), 0.0, abs_tol=1e-5)
    assert math.isclose(float(gw.float().abs().max()), 0.0, abs_tol=1e-5)
