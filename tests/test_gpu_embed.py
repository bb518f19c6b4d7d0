"""dv_embed (bit for bit) and its gradient against their 64-bit forms; every
sort path, runs of one token across chunks, accumulation; refusals."""
import math

import numpy as np
import pytest
import torch

from tests.train_common import check, embed_backward_reference

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def tokens(rng, N, V, how):
    if how == "one":
        ids = np.full(N, V // 2)
    elif how == "few":
        ids = rng.integers(0, min(V, 3), N)
    elif how == "frequent":
        ids = np.minimum(V ** rng.random(N) - 1, V - 1).astype(np.int64)
    else:
        ids = rng.integers(0, V, N)
    ids = ids.astype(np.int32)
    if how != "one":
        ids[rng.random(N) < 0.05] = -1
        ids[rng.random(N) < 0.02] = V
    return torch.from_numpy(ids)


def strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    view = wide[:, pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t)
    return view


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V", [(1, 1, 1), (1, 4096, 100), (5, 3, 10), (64, 64, 1000), (33, 77, 500), (1000, 130, 301)])
def test_lookup(dv, N, D, V, dtype):
    print(f"embed N={N} D={D} V={V} {dtype}", flush=True)
    rng = np.random.default_rng(N + D + V)
    w = torch.from_numpy(rng.normal(size=(V, D))).to(dtype)
    ids = tokens(rng, N, V, "any")
    ok = (ids >= 0) & (ids < V)
    for scale in (1.0, math.sqrt(D), -0.125):
        want = torch.where(ok[:, None], w[ids.clamp(0, V - 1).long()].float() * torch.tensor(scale, dtype=torch.float32),
                           torch.zeros(())).to(dtype)
        for pad in (0, 3, 8):
            got = dv.embed(strided(w, pad), ids.to(DEV), scale=scale)
            assert torch.equal(got.cpu(), want)


# rows below and above what one block sorts, tokens of one to five digits
CASES = [(1, 8, 1, "any"), (3, 5, 7, "any"), (100, 64, 63, "any"), (257, 33, 64, "few"), (1000, 128, 5000, "frequent"),
         (8192, 16, 300, "frequent"), (8193, 8, 70000, "any"), (20000, 24, 4097, "frequent"), (9000, 8, 300000, "frequent"),
         (300, 40, 9, "one"), (40000, 8, 11, "one"), (70000, 4, 1000, "few")]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,D,V,how", CASES)
def test_gradient(dv, N, D, V, how, dtype):
    print(f"embed backward N={N} D={D} V={V} {how} {dtype}", flush=True)
    rng = np.random.default_rng(N + D + V)
    ids = tokens(rng, N, V, how)
    grad = torch.from_numpy(rng.normal(size=(N, D))).to(dtype)
    base = torch.from_numpy(rng.normal(size=(V, D))).to(dtype)
    for pad, scale in ((0, 1.0), (5, 3.5)):
        want, tol = embed_backward_reference(grad, ids, V, scale)
        gd = strided(grad, pad)
        got = dv.embed_backward(gd, ids.to(DEV), V, scale=scale)
        check(got, want, tol, "grad")
        again = dv.embed_backward(gd, ids.to(DEV), V, scale=scale, grad_weight=torch.full_like(got, 9.0))
        assert torch.equal(got, again)
        want, tol = embed_backward_reference(grad, ids, V, scale, base)
        acc = base.to(DEV)
        assert dv.embed_backward(gd, ids.to(DEV), V, scale=scale, grad_weight=acc, accumulate=True) is acc
        check(acc, want, tol, "accumulated")
        absent = torch.ones(V, dtype=torch.bool)
        absent[ids[(ids >= 0) & (ids < V)].long()] = False
        assert torch.equal(acc.cpu()[absent], base[absent])
        assert not got[absent.to(DEV)].any()


def test_a_single_block_of_every_row_count(dv):
    """Row counts around a wave's, a chunk's and a block's share of the sort."""
    rng = np.random.default_rng(1)
    for N in (2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 511, 512, 513, 1023, 1024, 1025, 8191):
        ids = tokens(rng, N, 50, "any")
        grad = torch.from_numpy(rng.normal(size=(N, 4))).float()
        want, tol = embed_backward_reference(grad, ids, 50, 1.0)
        check(dv.embed_backward(grad.to(DEV), ids.to(DEV), 50), want, tol, f"N={N}")


def test_no_rows(dv):
    g = torch.empty((0, 6), dtype=torch.bfloat16, device=DEV)
    ids = torch.empty(0, dtype=torch.int32, device=DEV)
    w = torch.ones((5, 6), dtype=torch.bfloat16, device=DEV)
    assert dv.embed(w, ids).shape == (0, 6)
    assert not dv.embed_backward(g, ids, 5).any()
    keep = dv.embed_backward(g, ids, 5, grad_weight=w, accumulate=True)
    assert bool((keep == 1).all())


def test_only_ids_that_are_no_token(dv):
    ids = torch.full((100,), -5, dtype=torch.int32, device=DEV)
    assert not dv.embed_backward(torch.ones((100, 8), device=DEV), ids, 5).any()
    assert not dv.embed(torch.ones((5, 8), device=DEV), ids).any()


def test_refusals(dv):
    w = torch.zeros((10, 8), device=DEV)
    ids = torch.zeros(4, dtype=torch.int32, device=DEV)
    for bad in (lambda: dv.embed(w.half(), ids), lambda: dv.embed(w, ids.long()), lambda: dv.embed(w.t(), ids),
                lambda: dv.embed(w, ids, out=torch.zeros((3, 8), device=DEV)),
                lambda: dv.embed_backward(w[:4], ids, 10, accumulate=True),
                lambda: dv.embed_backward(w[:3], ids, 10),
                lambda: dv.embed_backward(w[:4], ids, 10, grad_weight=torch.zeros((9, 8), device=DEV))):
        with pytest.raises((TypeError, ValueError)):
            bad()
    for bad in (lambda: dv.embed(w, ids, scale=math.inf), lambda: dv.embed(w, ids, out=w[:4]),
                lambda: dv.embed_backward(w[:4], ids, 10, scale=math.nan),
                lambda: dv.embed_backward(w[:4], ids, 10, grad_weight=w)):
        with pytest.raises(dv.DvError):
            bad()


def test_ids_that_are_no_vector_are_refused(dv):
    w = torch.zeros((10, 8), device=DEV)
    for ids in (torch.tensor(3, dtype=torch.int32, device=DEV), torch.zeros((2, 2), dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError):
            dv.embed(w, ids)
        with pytest.raises(ValueError):
            dv.embed_backward(w[:2], ids, 10)
