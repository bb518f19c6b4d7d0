"""dv_distill_loss and its gradient against their 64-bit forms, element by
element within derived bounds; edges of masks, lists and logits; refusals."""
import math

import numpy as np
import pytest
import torch

from tests.train_common import check, distill_reference, masks, pack_mask, row_mask
from tests.train_common import U, UB

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def make(seed, N, V, K, dtype, S, shares=(0.0, 0.01, 0.5, 1.0)):
    rng = np.random.default_rng(seed)
    z = torch.from_numpy(rng.normal(size=(N, V)) * 3).to(dtype)
    may = masks(rng, S, V, shares) if S else None
    states = torch.from_numpy(rng.integers(-1, S + 1, N).astype(np.int32)) if S else None
    mask = row_mask(may, states, N, V)
    ids = torch.from_numpy(rng.integers(-1, V + 1, (N, K)).astype(np.int32))
    for n in range(N):  # most entries allowed, one of them twice
        allowed = torch.nonzero(mask[n])[:, 0]
        if allowed.numel():
            k = rng.integers(0, K, K // 2 + 1)
            ids[n, k] = allowed[rng.integers(0, allowed.numel(), len(k))].int()
        ids[n, K - 1] = ids[n, 0]
    top = torch.from_numpy(rng.normal(size=(N, K)) * 3).float()
    top[:, K // 2] = -math.inf if K > 2 else 0.0
    g = torch.from_numpy(rng.normal(size=N)).float()
    return z, ids, top, may, states, mask, g


def on_device(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    view = wide[:, pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t)
    return view


def run(dv, z, ids, top, c, may, states, g, pad=0, in_place=False):
    kw = dict(inv_temperature=c)
    if may is not None:
        kw.update(allow=pack_mask(may).to(DEV), states=states.to(DEV))
    zd = on_device(z, pad)
    args = (zd, ids.to(DEV), top.to(DEV))
    alone = dv.distill_loss(*args, **kw)
    loss, grad = dv.distill_loss_backward(*args, g.to(DEV), grad=zd if in_place else None, **kw)
    torch.cuda.synchronize()
    return alone, loss, grad


SIZES = [(1, 1, 1), (1, 7, 3), (2, 8, 1), (3, 33, 5), (5, 1000, 20), (4, 4099, 64), (2, 70001, 100), (1, 128256, 1024),
         (260, 500, 9), (300, 5001, 33)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_matches_the_64_bit_form(dv, N, V, K, dtype, masked):
    print(f"distill N={N} V={V} K={K} {dtype} masked={masked}", flush=True)
    z, ids, top, may, states, mask, g = make(N + V + K, N, V, K, dtype, 5 if masked else 0)
    for c, pad, in_place in ((1.0, 0, False), (0.5, 3, True), (1.25, 8, False)):
        ref = distill_reference(z, ids, top, c, mask, g)
        alone, loss, grad = run(dv, z, ids, top, c, may, states, g, pad, in_place)
        check(loss, ref["loss"], ref["loss_tol"], "loss")
        check(alone, ref["loss"], ref["loss_tol"], "loss alone")
        check(grad, ref["grad"], ref["grad_tol"], "grad")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [3, 300])
def test_masked_places_and_lowest_values(dv, dtype, N):
    """NaN and infinities in masked places; rows masked by the type's lowest
    value instead of a table; rows with nothing left."""
    V, K = 1003, 6
    z, ids, top, may, states, mask, g = make(9, N, V, K, dtype, 2, shares=(0.4,))
    states[:] = 0
    mask = row_mask(may, states, N, V)
    ids[:, :] = torch.nonzero(may[0])[:6, 0].int()
    ref = distill_reference(z, ids, top, 1.0, mask, g)
    dirty = z.clone()
    hidden = torch.nonzero(~may[0])[:, 0]
    dirty[:, hidden[0::3]] = float("nan")
    dirty[:, hidden[1::3]] = math.inf
    dirty[:, hidden[2::3]] = -math.inf
    _, loss, grad = run(dv, dirty, ids, top, 1.0, may, states, g)
    check(loss, ref["loss"], ref["loss_tol"], "loss")
    check(grad, ref["grad"], ref["grad_tol"], "grad")
    # the type's lowest value where the table would mask: no table, the same distribution
    low = torch.where(mask, z, torch.tensor(torch.finfo(dtype).min, dtype=dtype))
    _, loss, grad = run(dv, low, ids, top, 1.0, None, None, g)
    check(loss, ref["loss"], ref["loss_tol"], "loss")
    check(grad, ref["grad"], ref["grad_tol"], "grad")
    # a row of nothing but the lowest value is uniform; of -infinity, empty
    flat = torch.full((N, V), torch.finfo(dtype).min, dtype=dtype)
    for c in (1.0, 2.0):
        r = distill_reference(flat, ids, top, c, torch.ones_like(mask), g)
        _, loss, grad = run(dv, flat, ids, top, c, None, None, g)
        check(loss, r["loss"], r["loss_tol"], "loss")
        check(grad, r["grad"], r["grad_tol"], "grad")
    _, loss, grad = run(dv, torch.full((N, V), -math.inf, dtype=dtype), ids, top, 1.0, None, None, g)
    assert not loss.any() and not grad.any()
    # an unmasked NaN is seen, wherever it is, also where every logit is NaN
    for at in (slice(0, 1), slice(V - 1, V), slice(0, V)):
        bad = z.clone()
        bad[1, at] = float("nan")
        alone, loss, grad = run(dv, bad, ids, top, 1.0, None, None, g)
        assert bool(torch.isnan(loss[1])) and bool(torch.isnan(alone[1]))
        assert bool(torch.isfinite(loss[0]))
    bad_top = top.clone()
    bad_top[1, 0] = float("nan")
    assert bool(torch.isnan(run(dv, z, ids, bad_top, 1.0, None, None, g)[1][1]))
    # nothing listed
    none = torch.full_like(ids, -1)
    _, loss, grad = run(dv, z, none, top, 1.0, None, None, g)
    assert not loss.any() and not grad.any()
    # a listed token that the model rules out: infinite loss, finite gradient
    out = z.clone()
    out[0, int(ids[0, 0])] = -math.inf
    _, loss, grad = run(dv, out, ids, top, 1.0, None, None, g)
    assert float(loss[0]) == math.inf and bool(torch.isfinite(grad).all())


def test_gradient_against_differences(dv):
    N, V, K = 4, 300, 12
    z, ids, top, may, states, mask, g = make(17, N, V, K, torch.float32, 3, shares=(0.5, 1.0))
    kw = dict(inv_temperature=0.7, allow=pack_mask(may).to(DEV), states=states.to(DEV))
    args = (ids.to(DEV), top.to(DEV))
    _, grad = dv.distill_loss_backward(z.to(DEV), *args, g.to(DEV), **kw)
    rng = np.random.default_rng(3)
    for _ in range(6):
        d = torch.from_numpy(rng.normal(size=z.shape)).float()
        h = 2.0 ** -6
        up, down = (dv.distill_loss((z + s * h * d).to(DEV), *args, **kw).cpu().double() for s in (1, -1))
        diff = float(((up - down) * g.double()).sum()) / (2 * h)
        along = float((grad.cpu().double() * d.double()).sum())
        assert abs(diff - along) < 0.005 * (1 + abs(along)), (diff, along)


def test_no_rows_and_same_bits(dv):
    z = torch.empty((0, 50), device=DEV)
    ids = torch.empty((0, 4), dtype=torch.int32, device=DEV)
    loss, grad = dv.distill_loss_backward(z, ids, ids.float(), torch.empty(0, device=DEV))
    assert loss.numel() == 0 and grad.numel() == 0
    z, ids, top, may, states, mask, g = make(23, 20, 40000, 50, torch.bfloat16, 4)
    a = run(dv, z, ids, top, 1.0, may, states, g)
    b = run(dv, z, ids, top, 1.0, may, states, g)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals(dv):
    z = torch.zeros((4, 100), device=DEV)
    ids = torch.zeros((4, 3), dtype=torch.int32, device=DEV)
    top = torch.zeros((4, 3), device=DEV)
    g = torch.zeros(4, device=DEV)
    for bad in (lambda: dv.distill_loss(z.half(), ids, top), lambda: dv.distill_loss(z, ids.long(), top),
                lambda: dv.distill_loss(z, ids, top.bfloat16()), lambda: dv.distill_loss(z, ids[:3], top[:3]),
                lambda: dv.distill_loss(z, ids, top[:, :2].contiguous()),
                lambda: dv.distill_loss(z, ids, top, states=torch.zeros(4, dtype=torch.int32, device=DEV)),
                lambda: dv.distill_loss_backward(z, ids, top, g[:3]),
                lambda: dv.distill_loss_backward(z, ids, top, g, grad=z.bfloat16())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    wide = torch.zeros((4, 130), device=DEV)
    for bad in (lambda: dv.distill_loss(z, ids, top, inv_temperature=0.0),
                lambda: dv.distill_loss(z, ids, top, inv_temperature=math.nan),
                lambda: dv.distill_loss(z, ids[:, :0].contiguous(), top[:, :0].contiguous()),
                lambda: dv.distill_loss_backward(wide[:, :100], ids, top, g, grad=wide[:, 1:101])):
        with pytest.raises(dv.DvError):
            bad()


def far_reference(z, ids, top, c, g):
    """distill_reference for unmasked rows at once, with bounds that do not grow
    with the tokens: a sum of terms of one sign is off by as many U of itself as its
    chain is long, at most 64 or V / 512 terms of a lane and fewer than 64 joins."""
    N, V = z.shape
    z64, t64 = z.double(), top.double()
    zc, tc = c * (z64 - z64.max(1, keepdim=True).values), c * (t64 - t64.max(1, keepdim=True).values)
    lnp = zc - torch.logsumexp(zc, 1, keepdim=True)
    lnq = tc - torch.logsumexp(tc, 1, keepdim=True)
    q, at = lnq.exp(), ids.long()
    span = lnq - lnp.gather(1, at)
    loss = (q * span).sum(1)
    # exp's argument (two roundings) and its own, the sums, the logarithms
    rel = U * (max(64, V / 512) + 64 + 8 * (zc.clamp(min=-120).abs() + math.log(V) + 4))
    loss_tol = (q * (rel.gather(1, at) + U * (64 + 8 * (tc.abs() + lnq.abs() + span.abs())))).sum(1)
    Q = torch.zeros_like(z64).scatter_add_(1, at, q)
    w = g.double()[:, None] * c
    y = w * (lnp.exp() - Q)
    store = UB if z.dtype == torch.bfloat16 else 2 * U
    tol = (w.abs() * (lnp.exp() * rel + Q * U * (96 + 16 * tc.abs().max())) + store * y.abs()) * 1.01 + 1e-37
    return loss, loss_tol, y, tol


# a block a row, rows split over blocks, rows held in registers
@pytest.mark.parametrize("N,V,dtype", [(6, 700, torch.float32), (6, 5000, torch.bfloat16), (7, 50000, torch.float32),
                                       (8500, 1001, torch.float32), (2200, 8191, torch.bfloat16), (170, 40000, torch.float32)])
@pytest.mark.parametrize("c", [1.0, 0.75])
def test_logits_far_from_zero(dv, N, V, dtype, c):
    """Rows whose logits lie about 1e4, 1e5 and 6e5 from zero, on both sides of
    it: a softmax knows differences only, which are exact there."""
    print(f"distill far N={N} V={V} {dtype} c={c}", flush=True)
    rng = np.random.default_rng(N + V)
    ulp = 2.0 ** 12 if dtype == torch.bfloat16 else 2.0 ** -4
    c2 = np.float32(c) * np.float32(1.4426950408889634)

    def rounding(m):  # of the largest logit's exponent of two, in units of e
        m = m.astype(np.float32)
        return (m.astype(np.float64) * np.float64(c2) - np.float64(m * c2)) * math.log(2)

    # of 64 values near each distance the one whose exponent rounds most
    some = np.array([1e4, 1e5, 6e5])[np.arange(N) % 3][:, None] * rng.uniform(0.9, 1.1, (N, 64))
    some = np.round(some / ulp) * ulp
    some[1::2] *= -1
    some = torch.from_numpy(some).to(dtype).double().numpy()
    far = some[np.arange(N), np.abs(rounding(some)).argmax(1)]
    step = rng.integers(0, 200, (N, V)) * (ulp if dtype == torch.bfloat16 else 0.125)
    step[:, ::2] = 0  # half of the tokens at the maximum
    z = torch.from_numpy(far[:, None] - step).to(dtype)
    assert dtype == torch.bfloat16 or bool((z.double() == torch.from_numpy(far[:, None] - step)).all())
    ids = torch.from_numpy(np.stack([rng.permutation(V)[:6] // 2 * 2 for _ in range(N)]).astype(np.int32))
    top = torch.from_numpy(rng.normal(size=(N, 6))).float()
    g = torch.from_numpy(rng.normal(size=N)).float()
    loss, loss_tol, grad, grad_tol = far_reference(z, ids, top, c, g)
    # what a first-order factor for that rounding would leave out passes the bound
    assert (rounding(far) ** 2 / 2 > 2 * loss_tol.numpy()).any()
    alone, got, got_grad = run(dv, z, ids, top, c, None, None, g)
    check(alone, loss, loss_tol, "loss alone")
    check(got, loss, loss_tol, "loss")
    check(got_grad, grad, grad_tol, "grad")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,V", [(4, 300), (2, 90000), (8500, 2001)])  # a block a row, split rows, held rows
def test_largest_inverse_temperature(dv, dtype, N, V):
    """Both softmaxes are one token each there: where it is the same one, nothing is left."""
    rng = np.random.default_rng(V)
    z = torch.from_numpy(rng.integers(-50, 50, (N, V))).to(dtype)
    best = torch.from_numpy(rng.integers(0, V, N))
    z[torch.arange(N), best] = 64.0
    ids = torch.stack([best, (best + 1) % V], 1).int()
    top = torch.tensor([[2.0, 1.0]]).repeat(N, 1)
    alone, loss, grad = run(dv, z, ids, top, 2.3e38, None, None, torch.full((N,), 0.5))
    assert not alone.any() and not loss.any() and not grad.any()
