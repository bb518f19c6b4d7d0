"""The calls from the last layer to the logits on the host (no GPU needed):
workspace queries, and arguments rejected before any HIP call.  Pointers are
fake: each call is built so that a check rejects it."""
import pytest
import torch

import paper_2403_06988_amd as dv

lib = dv.lib
OK, INVALID, SHAPE, DTYPE, ALIAS, WORKSPACE, HIP = range(7)
P = 0x7F0000000000
GB = 1 << 30
BIG = 1 << 50


def norm(x=P, ldx=64, res=P + GB, ldr=64, w=P + 2 * GB, dt=1, N=8, D=64, eps=1e-6, total=P + 3 * GB, out=P + 4 * GB,
         rstd=P + 5 * GB, q=P + 6 * GB, s=P + 7 * GB):
    return lib.dv_rms_norm(x, ldx, res, ldr, w, dt, N, D, eps, total, out, rstd, q, s, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID),
    (dict(out=None, q=None, s=None), INVALID), (dict(x=P + 1), INVALID), (dict(res=P + GB + 1), INVALID),
    (dict(w=P + 2 * GB + 2, dt=0), INVALID), (dict(total=P + 3 * GB + 1), INVALID), (dict(out=P + 4 * GB + 1), INVALID),
    (dict(q=P + 6 * GB + 4), INVALID), (dict(s=P + 7 * GB + 2), INVALID),
    (dict(N=-1), SHAPE), (dict(N=(1 << 20) + 1), SHAPE), (dict(D=0), SHAPE), (dict(D=65537, ldx=70000, ldr=70000), SHAPE),
    (dict(ldx=63), SHAPE), (dict(ldr=63), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(eps=float("inf")), SHAPE), (dict(dt=2), DTYPE),
    (dict(out=P), ALIAS), (dict(out=P + GB), ALIAS), (dict(rstd=P + 16), ALIAS), (dict(q=P + GB + 8), ALIAS),
    (dict(s=P + 4), ALIAS), (dict(total=P + 2), ALIAS), (dict(total=P + GB + 64), ALIAS), (dict(total=P, ldx=65), ALIAS),
    (dict(total=P + GB, ldr=72), ALIAS), (dict(total=P + 4 * GB + 64), ALIAS), (dict(out=P + 2 * GB), ALIAS),
    (dict(s=P + 6 * GB + 64), ALIAS), (dict(total=P, res=P + 64), ALIAS),
])
def test_rms_norm_rejects_before_launch(kw, status):
    assert norm(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_rms_norm:")


def norm_back(g=P, ldg=64, h=P + GB, ldh=64, w=P + 2 * GB, r=P + 3 * GB, gt=P + 4 * GB, ldgt=64, dt=1, N=8, D=64,
              gx=P + 5 * GB, gw=P + 6 * GB, ws=P + 7 * GB, nb=BIG):
    return lib.dv_rms_norm_backward(g, ldg, h, ldh, w, r, gt, ldgt, dt, N, D, gx, gw, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(g=None), INVALID), (dict(h=None), INVALID), (dict(w=None), INVALID), (dict(r=None), INVALID),
    (dict(gx=None, gw=None), INVALID), (dict(g=P + 1), INVALID), (dict(h=P + GB + 1), INVALID), (dict(gt=P + 4 * GB + 1), INVALID),
    (dict(gx=P + 5 * GB + 1), INVALID), (dict(gw=P + 6 * GB + 2, dt=0), INVALID),
    (dict(N=-1), SHAPE), (dict(D=0), SHAPE), (dict(ldg=63), SHAPE), (dict(ldh=63), SHAPE), (dict(ldgt=63), SHAPE),
    (dict(dt=7), DTYPE), (dict(ws=None), WORKSPACE), (dict(nb=64), WORKSPACE), (dict(ws=P + 7 * GB + 8), WORKSPACE),
    (dict(gx=P), ALIAS), (dict(gx=P + GB), ALIAS), (dict(gx=P + 4 * GB), ALIAS), (dict(gw=P + 2 * GB), ALIAS),
    (dict(gw=P + 5 * GB + 64), ALIAS), (dict(ws=P + 3 * GB), ALIAS), (dict(ws=P + 6 * GB), ALIAS),
])
def test_rms_norm_backward_rejects_before_launch(kw, status):
    assert norm_back(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_rms_norm_backward:")


def quantize(x=P, ld=200, dt=1, N=300, K=200, tile=1, q=P + GB, s=P + 2 * GB, tq=P + 3 * GB, ts=P + 4 * GB):
    return lib.dv_quantize_f8(x, ld, dt, N, K, tile, q, s, tq, ts, None)


@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(tq=None), INVALID), (dict(ts=None), INVALID),
    (dict(q=None, s=None, tq=None, ts=None), INVALID), (dict(x=P + 1), INVALID), (dict(q=P + GB + 8), INVALID),
    (dict(tq=P + 3 * GB + 8), INVALID), (dict(s=P + 2 * GB + 1), INVALID), (dict(ts=P + 4 * GB + 2), INVALID),
    (dict(N=-1), SHAPE), (dict(N=(1 << 24) + 1), SHAPE), (dict(K=0), SHAPE), (dict(ld=199), SHAPE), (dict(tile=0), SHAPE),
    (dict(tile=64), SHAPE), (dict(N=1 << 24, K=1 << 14, ld=1 << 14), SHAPE), (dict(dt=5), DTYPE),
    (dict(q=P), ALIAS), (dict(s=P + 64), ALIAS), (dict(tq=P + GB + 16), ALIAS), (dict(ts=P + 2 * GB + 4), ALIAS),
    (dict(tq=P + GB + 300 * 256 - 16), ALIAS),
])
def test_quantize_rejects_before_launch(kw, status):
    assert quantize(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_quantize_f8:")


def product(a=P, lda=256, sa=P + GB, b=P + 2 * GB, ldb=256, sb=P + 3 * GB, tile=128, M=8, N=300, K=256, dt=1, out=P + 4 * GB,
            ldo=300, ws=P + 5 * GB, nb=BIG):
    return lib.dv_product_f8(a, lda, sa, b, ldb, sb, tile, M, N, K, dt, out, ldo, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(a=None), INVALID), (dict(sa=None), INVALID), (dict(b=None), INVALID), (dict(sb=None), INVALID), (dict(out=None), INVALID),
    (dict(a=P + 8), INVALID), (dict(b=P + 2 * GB + 8), INVALID), (dict(out=P + 4 * GB + 1), INVALID),
    (dict(sa=P + GB + 2), INVALID), (dict(sb=P + 3 * GB + 1), INVALID),
    (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(M=1 << 20, N=1 << 16, ldo=1 << 16), SHAPE), (dict(K=0), SHAPE),
    (dict(K=200), SHAPE), (dict(K=(1 << 22) + 128, lda=1 << 23, ldb=1 << 23), SHAPE), (dict(lda=255), SHAPE), (dict(ldb=240), SHAPE),
    (dict(lda=264), SHAPE), (dict(ldb=257), SHAPE), (dict(ldb=(1 << 22) + 16), SHAPE), (dict(ldo=299), SHAPE), (dict(tile=2), SHAPE),
    (dict(dt=2), DTYPE),
    (dict(out=P + 16), ALIAS), (dict(out=P + GB), ALIAS), (dict(out=P + 2 * GB + 64), ALIAS), (dict(out=P + 3 * GB), ALIAS),
])
def test_product_rejects_before_launch(kw, status):
    assert product(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_product_f8:")


def test_product_workspace():
    """None of a shape, or a size that a call insists on."""
    q = lib.dv_product_f8_workspace_bytes
    assert q(-1, 8, 128) == q(8, 0, 128) == q(8, 8, 100) == q(8, 8, 0) == q(1 << 20, 1 << 16, 128) == 0
    for M, N, K in ((8, 256, 1 << 17), (100, 1000, 1 << 16), (1, 128256, 4096), (8192, 32000, 4096), (4096, 4096, 128256)):
        need = q(M, N, K)
        assert need <= 16 * M * N * 4 + 256
        if need:
            kw = dict(M=M, N=N, K=K, lda=K, ldb=K, ldo=N, b=P + 20 * GB, sb=P + 40 * GB, out=P + 60 * GB, ws=P + 80 * GB)
            assert product(**kw, nb=need - 1) == product(**dict(kw, ws=None)) == product(**dict(kw, ws=P + 80 * GB + 8)) == WORKSPACE
            assert product(**dict(kw, ws=P + 60 * GB)) == ALIAS


def adjust(z=P, ld=1000, dt=1, N=8, V=1000, h=P + GB, ldh=50, H=50, le=P + 2 * GB, pr=P + 3 * GB, rep=P + 4 * GB, pre=P + 5 * GB,
           fr=P + 6 * GB, ids=P + 7 * GB, bias=P + 8 * GB, nb=4, al=P + 9 * GB, S=2, st=P + 10 * GB, out=P + 11 * GB, ldo=1000):
    return lib.dv_adjust_logits(z, ld, dt, N, V, h, ldh, H, le, pr, rep, pre, fr, ids, bias, nb, al, S, st, out, ldo, None)


@pytest.mark.parametrize("kw,status", [
    (dict(z=None), INVALID), (dict(out=None), INVALID), (dict(h=None), INVALID), (dict(le=None), INVALID), (dict(ids=None), INVALID),
    (dict(bias=None), INVALID), (dict(al=None), INVALID), (dict(st=None), INVALID), (dict(z=P + 1), INVALID),
    (dict(out=P + 11 * GB + 2, dt=0), INVALID),
    (dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(ld=999), SHAPE), (dict(ldo=999), SHAPE), (dict(ldh=49), SHAPE), (dict(H=-1), SHAPE),
    (dict(H=1 << 20, ldh=1 << 20), SHAPE), (dict(nb=-1), SHAPE), (dict(nb=1025), SHAPE), (dict(S=0), SHAPE),
    (dict(N=1 << 20, V=200000, ld=200000, ldo=200000), SHAPE), (dict(dt=9), DTYPE),
    (dict(out=P + 2), ALIAS), (dict(out=P, ldo=1001), ALIAS), (dict(out=P + GB), ALIAS), (dict(out=P + 2 * GB), ALIAS),
    (dict(out=P + 3 * GB), ALIAS), (dict(out=P + 4 * GB), ALIAS), (dict(out=P + 5 * GB), ALIAS), (dict(out=P + 6 * GB), ALIAS),
    (dict(out=P + 7 * GB), ALIAS), (dict(out=P + 8 * GB), ALIAS), (dict(out=P + 9 * GB), ALIAS), (dict(out=P + 10 * GB), ALIAS),
])
def test_adjust_rejects_before_launch(kw, status):
    assert adjust(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_adjust_logits:")


def test_no_rows_enqueue_nothing():
    assert norm(N=0, x=None, res=None, total=None, out=None, q=None, s=None) == OK
    assert norm_back(N=0, g=None, h=None, r=None, gt=None, gx=None, gw=None) == OK
    assert quantize(N=0, x=None, q=None, s=None, tq=None, ts=None) == OK
    assert product(M=0, a=None, sa=None, out=None) == OK
    assert adjust(N=0, z=None, out=None, h=None, le=None, ids=None, bias=None, st=None) == OK


def test_workspace_queries_never_fall_as_rows_grow():
    q = lib.dv_rms_norm_backward_workspace_bytes
    assert q(-1, 64) == q(8, 0) == q(8, 65537) == q((1 << 20) + 1, 64) == 0
    for D in (1, 64, 4096, 8193, 65536):
        sizes = [q(n, D) for n in (0, 1, 2, 100, 255, 256, 257, 1000, 1024, 1025, 8192, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_the_binding_checks_its_tensors():
    x = torch.zeros((4, 128))
    w = torch.ones(128)
    for call in (lambda: dv.rms_norm(x, w), lambda: dv.rms_norm_f8(x, w), lambda: dv.quantize_f8(x), lambda: dv.adjust_logits(x),
                 lambda: dv.rms_norm_backward(x, x, w, w),
                 lambda: dv.product_f8(x.to(dv.F8), w, x.to(dv.F8), w)):
        with pytest.raises(ValueError):
            call()
