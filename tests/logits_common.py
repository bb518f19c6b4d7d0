"""Plain forms of the operators between the last layer and the logits (torch on
the CPU, from their formulas in 64 bits), and the error bounds that the GPU
tests hold the kernels to.

U is the unit roundoff of fp32, UB that of bf16, U8 that of e4m3 (4 significant
bits; below 2^-6 its steps are 2^-9)."""
import math

import torch

U = 2.0 ** -24
UB = 2.0 ** -8
U8 = 2.0 ** -4
B = 128


def up(n):
    return (n + B - 1) // B * B


def own_rounding(dtype):
    return U if dtype == torch.float32 else UB


def blocks_of(x, tile):
    """x [n][k] with zeros up to whole blocks: by rows [n][kb][128], by tiles [nb][128][kb][128]."""
    n, k = x.shape
    p = torch.zeros((up(n) if tile != 1 else n, up(k)), dtype=x.dtype)
    p[:n, :k] = x
    return p.view(n, -1, B) if tile == 1 else p.view(p.shape[0] // B, B, p.shape[1] // B, B)


def quantize(x, tile):
    """The definition, bit for bit: (q [n][up(k)] float8_e4m3fn, scales as stored).  Each
    step is an fp32 operation that rounds once, as numpy and torch have them on the CPU."""
    n = x.shape[0]
    p = blocks_of(x.float(), tile)
    over = 2 if tile == 1 else (1, 3)
    bad = ~torch.isfinite(p).all(dim=2, keepdim=True) if tile == 1 else (~torch.isfinite(p)).any(3, True).any(1, True)
    clean = torch.where(torch.isfinite(p), p, torch.zeros(()))
    scale = clean.abs().amax(over, keepdim=True).clamp(min=2.0 ** -100) / torch.tensor(448.0)
    q = (clean / scale).to(torch.float8_e4m3fn).view(torch.uint8)
    q = torch.where(bad, torch.tensor(0x7F, dtype=torch.uint8), q)
    scale = torch.where(bad, torch.tensor(math.nan), scale)
    if tile == 1:
        return q.reshape(n, -1).view(torch.float8_e4m3fn), scale[:, :, 0].t().contiguous()
    return q.reshape(-1, p.shape[2] * B)[:n].view(torch.float8_e4m3fn), scale[:, 0, :, 0].contiguous()


def values(q, scales, tile):
    """What an operand stands for, [n][K] float64."""
    n, K = q.shape
    s = scales.double()
    s = s.t() if tile == 1 else s.repeat_interleave(B, 0)[:n]
    return q.float().double() * s.repeat_interleave(B, 1)


def product_reference(a, sa, b, sb, tile, dtype):
    """(a b^T, its bound).  A block's 128 products are exact, their sum in the matrix
    instruction loses at most 2 U of what it adds up to per addition; then one
    product with the scales (two roundings) and one addition a block.  bf16 results of
    more than 256 rows: the 8-bit matrix instruction cuts eight neighbouring products to
    13 bits below the largest of them, seven of them off by 2^-13 of it each at most."""
    va, vb = values(a, sa, 1), values(b, sb, tile)
    y = va @ vb.t()
    mag = va.abs() @ vb.abs().t()
    tol = (2 * B + a.shape[1] // B + 4) * U * mag + own_rounding(dtype) * y.abs()
    if dtype == torch.bfloat16 and a.shape[0] > 256:
        tol = tol + 7 * 2.0 ** -13 * mag
    return y, tol * 1.01 + 1e-37


# a row's sum of squares or products: 64 terms a lane at most, 6 additions in a wave, 16 waves
DEPTH = 64 + 6 + 16


def norm_reference(x, residual, weight, eps):
    """dict of results and bounds, float64; h exactly (its rounding is the type's)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    hd, w = h.double(), weight.double()
    D = x.shape[1]
    rstd = 1.0 / torch.sqrt((hd * hd).mean(1) + eps)
    # positive terms; the division, eps, root and reciprocal, each within 2 U of its result
    r_rel = (DEPTH * 0.5 + 6) * U
    y = hd * rstd[:, None] * w
    y_err = y.abs() * (r_rel + 2 * U) * 1.01 + 1e-37
    return dict(h=h, rstd=rstd, rstd_tol=rstd * r_rel * 1.01, y=y, y_err=y_err,
                out_tol=y_err + own_rounding(x.dtype) * y.abs() * 1.01)


def norm_backward_reference(g, h, weight, rstd, gt):
    """(grad_x, bound, grad_weight, bound); rstd as it is given (fp32)."""
    N, D = h.shape
    ulp = own_rounding(h.dtype)
    gd, hd, w, r = g.double(), h.double(), weight.double(), rstd.double()[:, None]
    gw = gd * w
    s = (gw * hd).sum(1, keepdim=True)
    mag = (gw * hd).abs().sum(1, keepdim=True)
    k, k_err = s / D * r ** 3, (mag * (DEPTH + 3) + s.abs() * 5) * U / D * r ** 3
    y = r * gw - hd * k
    err = 3 * U * (r * gw).abs() + hd.abs() * (k_err + 2 * U * k.abs())
    if gt is not None:
        y = y + gt.double()
        err = err + 2 * U * (gt.double().abs() + y.abs())
    dx_tol = (err + U * y.abs() + ulp * y.abs()) * 1.01 + 1e-37
    terms = gd * hd * r
    dw = terms.sum(0)
    dw_tol = ((N + 20) * U * terms.abs().sum(0) + ulp * dw.abs()) * 1.01 + 1e-37
    return y, dx_tol, dw, dw_tol


def adjust_reference(z, history=None, lengths=None, prompts=None, repetition=None, presence=None, frequency=None,
                     bias_ids=None, bias=None, may=None):
    """(float64 result, bound, which logits keep their bits); may [B][V] truth values."""
    Bn, V = z.shape
    out = z.double().clone()
    err = torch.zeros(out.shape, dtype=torch.float64)
    named = torch.zeros(out.shape, dtype=torch.bool)
    for n in range(Bn):
        if history is not None:
            length = max(0, min(int(lengths[n]), history.shape[1]))
            prompt = 0 if prompts is None else int(prompts[n])
            rho = 1.0 if repetition is None else float(repetition[n])
            p = 0.0 if presence is None else float(presence[n])
            f = 0.0 if frequency is None else float(frequency[n])
            seen, count = {}, {}
            for i, v in enumerate(history[n, :length].tolist()):
                if 0 <= v < V:
                    seen[v] = True
                    if i >= prompt:
                        count[v] = count.get(v, 0) + 1
            for v in seen:
                x = float(out[n, v])
                x = x / rho if x > 0 else x * rho
                c = count.get(v, 0)
                e = U * abs(x) if math.isfinite(x) else 0.0
                if c:
                    e += 3 * U * (abs(x) + abs(c * f) + abs(p)) if math.isfinite(x) else 0.0
                    x = x - c * f - p
                out[n, v], err[n, v], named[n, v] = x, e, True
        if bias_ids is not None:
            ids, b = bias_ids[n].tolist(), bias[n].tolist()
            total, mag, times = {}, {}, {}
            for v, x in zip(ids, b):
                if 0 <= v < V:
                    total[v] = total.get(v, 0.0) + x
                    mag[v] = mag.get(v, 0.0) + abs(x)
                    times[v] = times.get(v, 0) + 1
            for v in total:
                x = float(out[n, v]) + total[v]
                if math.isfinite(x):
                    err[n, v] += U * (abs(x) + (times[v] + 1) * mag[v])
                out[n, v], named[n, v] = x, True
    if may is not None:
        out[~may] = -math.inf
    tol = (err + own_rounding(z.dtype) * torch.where(torch.isfinite(out), out.abs(), torch.zeros(()).double())) * 1.01 + 1e-37
    tol[~named] = 0
    return out, tol, ~named
