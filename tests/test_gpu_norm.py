"""RMS norm with the residual's addition (in the type and in 8 bits) and its
gradients, against the formulas in 64 bits and against differences."""
import math

import numpy as np
import pytest
import torch

from tests.logits_common import B, U8, norm_backward_reference, norm_reference, up, values
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


def rows(rng, N, D, dtype, pad=0, scale=1.0, shift=0):
    """[N][D] on the device, rows D + pad apart, the first `shift` elements into its buffer; and on the CPU."""
    t = torch.from_numpy(rng.normal(size=(N, D)) * scale).to(dtype)
    buf = torch.full((N * (D + pad) + shift + 8,), 7.0, dtype=dtype, device=DEV)
    view = buf[shift:shift + N * (D + pad)].view(N, D + pad)[:, :D]
    view.copy_(t)
    return view, t


SIZES = [(1, 1), (1, 128), (3, 127), (2, 129), (1, 1024), (5, 1000), (300, 513), (7, 1025), (4, 2049), (3, 4096), (2, 4104),
         (2, 8200), (2, 16392), (2, 32776), (1, 65536), (1030, 64)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,D", SIZES)
def test_forward(dv, N, D, dtype):
    rng = np.random.default_rng(N * 70001 + D)
    pad, shift = (0, 0) if D % 8 == 0 else (3, 1)
    x, xc = rows(rng, N, D, dtype, pad, 1.0, shift)
    res, rc = rows(rng, N, D, dtype, 2 * pad, 3.0)
    w, wc = rows(rng, 1, D, dtype)
    w, wc = w[0].contiguous(), wc[0]
    for residual, resc in ((res, rc), (None, None)):
        want = norm_reference(xc, resc, wc, 1e-5)
        out, total, rstd = dv.rms_norm(x, w, 1e-5, residual=residual, want_rstd=True)
        check(out, want["y"], want["out_tol"], "out")
        check(rstd, want["rstd"], want["rstd_tol"], "rstd")
        if residual is not None:
            assert torch.equal(total.cpu(), want["h"])
        else:
            assert total is None
        q, scales, total8 = dv.rms_norm_f8(x, w, 1e-5, residual=residual)
        assert q.shape == (N, up(D)) and scales.shape == (up(D) // B, N)
        assert (total8 is None) == (residual is None) and (total8 is None or torch.equal(total8, total))
        q, scales = q.cpu(), scales.cpu()
        assert (q.view(torch.uint8)[:, D:] & 0x7F == 0).all()
        y = torch.zeros((N, up(D)), dtype=torch.float64)
        y[:, :D], err = want["y"], want["y_err"]
        exact = y.view(N, -1, B).abs().amax(2).clamp(min=2.0 ** -100) / 448
        # the largest element's error, and the division's rounding
        rel = float((err / want["y"].abs().clamp(min=1e-30)).max()) + 2.0 ** -23
        assert ((scales.t().double() - exact).abs() <= rel * exact).all()
        stands = values(q, scales, 1)[:, :D]
        step = torch.maximum(U8 * want["y"].abs(), 2.0 ** -10 * exact.repeat_interleave(B, 1)[:, :D])
        check(stands, want["y"], step * 1.01 + 4 * err, "8 bits")


def test_total_in_place(dv):
    rng = np.random.default_rng(3)
    x, xc = rows(rng, 33, 520, BF)
    res, rc = rows(rng, 33, 520, BF)
    x, res = x.contiguous(), res.contiguous()
    w = torch.ones(520, dtype=BF, device=DEV)
    out, total, _ = dv.rms_norm(x, w, residual=res)
    r2, x2 = res.clone(), x.clone()
    out2, t2, _ = dv.rms_norm(x, w, residual=r2, total=r2)
    out3, t3, _ = dv.rms_norm(x2, w, residual=res, total=x2)
    assert t2.data_ptr() == r2.data_ptr() and torch.equal(t2, total) and torch.equal(t3, total)
    assert torch.equal(out, out2) and torch.equal(out, out3)
    q, s, t4 = dv.rms_norm_f8(x, w, residual=res.clone())
    r5 = res.clone()
    q5, s5, t5 = dv.rms_norm_f8(x, w, residual=r5, total=r5)
    assert torch.equal(q.view(torch.uint8), q5.view(torch.uint8)) and torch.equal(s, s5) and torch.equal(t4, t5)


@pytest.mark.parametrize("D", [256, 2304])
def test_special_values(dv, D):
    """Zeros, an infinity, a NaN, rows near the type's largest and smallest: each row by itself."""
    x = torch.from_numpy(np.random.default_rng(5).normal(size=(7, D))).float()
    x[0] = 0
    x[1, 130] = math.inf
    x[2, 5] = math.nan
    x[3] *= 1e18            # squares up to 1e37
    x[4] *= 1e-18           # squares below the smallest normal number
    x[5] = 0
    x[5, 3] = 2.5
    w = torch.ones(D)
    out, _, rstd = dv.rms_norm(x.to(DEV), w.to(DEV), 1e-5, want_rstd=True)
    out = out.cpu()
    assert (out[0] == 0).all() and abs(float(rstd[0]) - 1e5 ** 0.5) < 1e-3
    assert torch.isnan(out[1, 130]) and (out[1, :130] == 0).all() and float(rstd[1]) == 0
    assert torch.isnan(out[2]).all()
    want = norm_reference(x[3:], None, w, 1e-5)
    check(out[3:], want["y"], want["out_tol"], "large, small and sparse rows")
    q, scales, _ = dv.rms_norm_f8(x.to(DEV), w.to(DEV), 1e-5)
    q, scales = q.cpu().view(torch.uint8), scales.cpu()
    assert (q[0] == 0).all() and torch.equal(scales[:, 0], torch.full((D // B,), 2.0 ** -100) / torch.tensor(448.0))
    assert (q[1, 128:256] == 0x7F).all() and torch.isnan(scales[1, 1]) and (q[1, :128] == 0).all()
    assert (q[2] == 0x7F).all() and torch.isnan(scales[:, 2]).all()
    assert torch.isfinite(scales[:, 3:]).all() and not (q[3:] & 0x7F == 0x7F).any()
    zero, _, _ = dv.rms_norm(x[:1].to(DEV), w.to(DEV), 0.0)
    assert torch.isnan(zero).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,D", SIZES + [(2500, 130), (1100, 1024)])
def test_backward(dv, N, D, dtype):
    rng = np.random.default_rng(N * 7001 + D)
    pad, shift = (0, 0) if D % 8 == 0 else (5, 1)
    h, hc = rows(rng, N, D, dtype, pad, 2.0, shift)
    g, gc = rows(rng, N, D, dtype, pad)
    gt, gtc = rows(rng, N, D, dtype, 0, 0.5, shift)
    w, wc = rows(rng, 1, D, dtype)
    w, wc = w[0].contiguous(), wc[0]
    rstd = (1.0 / torch.sqrt((hc.double() ** 2).mean(1) + 1e-5)).float()
    for grad_total, gtotal in ((gt, gtc), (None, None)):
        dx, dx_tol, dw, dw_tol = norm_backward_reference(gc, hc, wc, rstd, gtotal)
        gx, gw = dv.rms_norm_backward(g, h, w, rstd.to(DEV), grad_total=grad_total)
        check(gx, dx, dx_tol, "grad_x")
        check(gw, dw, dw_tol, "grad_weight")
        only_x, none = dv.rms_norm_backward(g, h, w, rstd.to(DEV), grad_total=grad_total, want_weight=False)
        none2, only_w = dv.rms_norm_backward(g, h, w, rstd.to(DEV), grad_total=grad_total, want_x=False)
        assert none is None and none2 is None and torch.equal(only_x, gx) and torch.equal(only_w, gw)


def test_no_rows(dv):
    x = torch.empty((0, 64), dtype=BF, device=DEV)
    w = torch.ones(64, dtype=BF, device=DEV)
    out, total, rstd = dv.rms_norm(x, w, residual=x, want_rstd=True)
    assert out.shape == total.shape == (0, 64) and rstd.shape == (0,)
    q, s, _ = dv.rms_norm_f8(x, w)
    assert q.shape == (0, 128) and s.shape == (1, 0)
    gw = torch.full((64,), 9.0, dtype=BF, device=DEV)
    gx, gw = dv.rms_norm_backward(x, x, w, rstd, grad_weight=gw)
    assert gx.shape == (0, 64) and (gw == 0).all()


def test_against_differences(dv):
    """d/dt of sum(g y(x + t v)) + sum(gt h) by central differences of the 64-bit form,
    against the kernel's gradients along v (and along u for the weight)."""
    rng = np.random.default_rng(11)
    N, D, eps = 6, 200, 1e-5
    x, w, g, gt, v = (torch.from_numpy(rng.normal(size=s)) for s in ((N, D), (D,), (N, D), (N, D), (N, D)))
    u = torch.from_numpy(rng.normal(size=D))

    def value(x, w):
        r = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
        return float((g * x * r * w).sum() + (gt * x).sum())

    f = lambda t: t.float().to(DEV)  # noqa: E731
    _, _, rstd = dv.rms_norm(f(x), f(w), eps, want_rstd=True)
    gx, gw = dv.rms_norm_backward(f(g), f(x), f(w), rstd, grad_total=f(gt))
    t = 1e-5
    along_x = (value(x + t * v, w) - value(x - t * v, w)) / (2 * t)
    along_w = (value(x, w + t * u) - value(x, w - t * u)) / (2 * t)
    # inputs rounded to fp32 and some 100 fp32 operations a term; the difference's own t^2 and 1e-16 / t terms are smaller
    size_x = float((gx.cpu().double().abs() * v.abs()).sum()) + 1
    size_w = float((gw.cpu().double().abs() * u.abs()).sum()) + 1
    assert abs(float((gx.cpu().double() * v).sum()) - along_x) < 1e-5 * size_x
    assert abs(float((gw.cpu().double() * u).sum()) - along_w) < 1e-5 * size_w


def test_every_result_of_one_call(dv):
    """The C call with both results, the sum over its residual and rstd: each as by itself."""
    rng = np.random.default_rng(12)
    N, D = 37, 700
    x, _ = rows(rng, N, D, BF)
    res, _ = rows(rng, N, D, BF)
    x, res, w = x.contiguous(), res.contiguous(), torch.ones(D, dtype=BF, device=DEV)
    out, total, rstd = dv.rms_norm(x, w, 1e-5, residual=res, want_rstd=True)
    q, scales, _ = dv.rms_norm_f8(x, w, 1e-5, residual=res)
    o2, r2, q2, s2 = (torch.empty_like(t) for t in (out, rstd, q, scales))
    st = dv.lib.dv_rms_norm(x.data_ptr(), D, res.data_ptr(), D, w.data_ptr(), dv.DV_BF16, N, D, 1e-5, res.data_ptr(),
                            o2.data_ptr(), r2.data_ptr(), q2.data_ptr(), s2.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert st == dv.DV_OK
    assert torch.equal(o2, out) and torch.equal(r2, rstd) and torch.equal(s2, scales) and torch.equal(res, total)
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8))


def test_a_row_added_to_itself_in_place(dv):
    x = torch.from_numpy(np.random.default_rng(13).normal(size=(9, 300))).float().to(DEV)
    w = torch.ones(300, device=DEV)
    want, total, _ = dv.rms_norm(x, w, residual=x)
    y = x.clone()
    out, t, _ = dv.rms_norm(y, w, residual=y, total=y)
    assert torch.equal(out, want) and torch.equal(t, total) and t.data_ptr() == y.data_ptr()
