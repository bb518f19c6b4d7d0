"""Plain 64-bit forms of the training operators (torch on the CPU, from their
formulas), and the error bounds that the GPU tests hold the kernels to.

U is the unit roundoff of fp32 (24 significant bits), UB that of bf16 (8).  A bound is a worst case, term by term:
a product's fp32 sum of n terms is off by at most n U times the sum of their
magnitudes, a stored result by its own rounding."""
import math

import numpy as np
import torch

U = 2.0 ** -24
UB = 2.0 ** -8


def pack_mask(may):
    """allow [S][ceil(V/32)] int32 of truth values [S][V]."""
    S, V = may.shape
    words = (V + 31) // 32
    bits = np.zeros((S, words * 32), bool)
    bits[:, :V] = may.numpy()
    packed = np.packbits(bits, axis=1, bitorder="little").view("<u4").astype("<u4").reshape(S, words)
    return torch.from_numpy(packed.view(np.int32).copy())


def row_mask(may, states, N, V):
    """[N][V] truth values: what each row's state allows."""
    if may is None:
        return torch.ones((N, V), dtype=torch.bool)
    out = torch.zeros((N, V), dtype=torch.bool)
    for n in range(N):
        s = int(states[n])
        if 0 <= s < may.shape[0]:
            out[n] = may[s]
    return out


def head_reference(x, w, targets, mask, grad_loss=None):
    """dict of the results and their bounds (``*_tol``), all float64."""
    N, D = x.shape
    V = w.shape[0]
    fp32 = x.dtype == torch.float32
    x, w = x.double(), w.double()
    z = x @ w.t()
    mag = x.abs() @ w.abs().t()
    # the product's sum (six of them for fp32's parts), and what the parts leave out
    z_err = ((6 if fp32 else 1) * (D + 64) * U + (2 * U if fp32 else 0)) * mag
    zm = torch.where(mask, z, torch.tensor(-math.inf, dtype=torch.float64))
    lse = torch.logsumexp(zm, 1)
    lse[~mask.any(1)] = -math.inf
    worst = torch.where(mask, z_err, torch.zeros(())).max(1).values
    top = torch.where(mask.any(1), zm.max(1).values, torch.zeros(()).double())
    spread = torch.where(mask, (top[:, None] - z).clamp(max=120.0), torch.zeros(()).double())
    # exp: its argument's two roundings, its own; then the sum of V terms
    exp_err = 4 * U * (spread.max(1).values + 4)
    finite_lse = torch.where(torch.isfinite(lse), lse, torch.zeros(()).double())
    lse_tol = worst + exp_err + (V + 64) * U + 4 * U * (finite_lse.abs() + top.abs() + 1)
    t = targets.long()
    part = (t >= 0) & (t < V)
    part = part & mask[torch.arange(N), t.clamp(0, V - 1)]
    zt = z[torch.arange(N), t.clamp(0, V - 1)]
    loss = torch.where(part, lse - zt, torch.zeros(()).double())
    loss_tol = lse_tol + worst + 4 * U * (zt.abs() + top.abs()) + 2 * U
    out = dict(loss=loss, loss_tol=loss_tol, lse=lse, lse_tol=lse_tol)
    if grad_loss is None:
        return out
    g = torch.where(part, grad_loss.double(), torch.zeros(()).double())
    p = torch.where(mask & part[:, None], torch.exp(zm - finite_lse[:, None]), torch.zeros(()).double())
    G = p.clone()
    G[torch.arange(N)[part], t[part]] -= 1.0
    # p's relative error: its logit's, the lse's, exp's own; the subtraction's and the weight's rounding
    rel = z_err + lse_tol[:, None] + 4 * U * (spread + 8)
    G_err = (p * rel * 1.1 + 2 * U * (p + G.abs())) * g.abs()[:, None]
    G = G * g[:, None]
    G_err = G_err + (2 * U if fp32 else UB) * G.abs()
    ulp = U if fp32 else UB
    for name, a, b, n in (("grad_x", G, w, V), ("grad_weight", G.t(), x, N)):
        err = G_err if name == "grad_x" else G_err.t()
        y = a @ b
        mags = a.abs() @ b.abs()
        out[name] = y
        out[name + "_tol"] = ((err @ b.abs()) + ((6 if fp32 else 1) * (n + 64) * U + (2 * U if fp32 else 0)) * mags
                              + ulp * y.abs()) * 1.01 + 1e-37
    return out


def distill_reference(z, ids, top, c, mask, grad_loss=None):
    N, V = z.shape
    bf16 = z.dtype == torch.bfloat16
    z, top = z.double(), top.double()
    loss, loss_tol = torch.zeros(N).double(), torch.zeros(N).double()
    grad = torch.zeros((N, V)).double()
    grad_tol = torch.zeros((N, V)).double()
    for n in range(N):
        A = torch.nonzero(mask[n])[:, 0]
        listed = [k for k in range(ids.shape[1])
                  if 0 <= int(ids[n, k]) < V and mask[n, int(ids[n, k])] and top[n, k] != -math.inf]
        if not listed or A.numel() == 0 or bool((z[n, A] == -math.inf).all()):
            continue
        k = torch.tensor(listed)
        at = ids[n, k].long()
        tk = top[n, k]
        q = torch.exp(c * (tk - tk.max()))
        lnq = c * (tk - tk.max()) - torch.log(q.sum())
        q = q / q.sum()
        zz = z[n, A]
        m = zz.max()
        e = torch.exp(c * (zz - m))
        lns = torch.log(e.sum())
        lnp = c * (z[n] - m) - lns
        live = q > 0
        loss[n] = (q[live] * (lnq[live] - lnp[at[live]])).sum()
        # each logarithm: a difference, a scaling, a sum's logarithm (V or K terms)
        span_z = (c * (m - z[n])).clamp(0, 200)
        ln_err = 6 * U * (span_z + lns.abs() + 2) + (V + 64) * U
        tq = 6 * U * (c * (tk.max() - tk)).clamp(0, 200) + (len(listed) + 64) * U * 2
        loss_tol[n] = (q * (ln_err[at] + tq * (1 + (lnq - lnp[at]).abs()) + 8 * U * (lnq.abs() + lnp[at].abs()))
                       )[live].sum() + len(listed) * U * (q * (lnq - lnp[at]).abs())[live].sum()
        if grad_loss is None:
            continue
        w = float(grad_loss[n]) * c
        p = torch.zeros(V).double()
        p[A] = torch.exp(lnp[A])
        Q = torch.zeros(V).double().index_add_(0, at, q)
        Q_err = torch.zeros(V).double().index_add_(0, at, q * (tq + 8 * U + len(listed) * U))
        y = w * (p - Q)
        y[~mask[n]] = 0
        grad[n] = y
        grad_tol[n] = (abs(w) * (p * (ln_err + 8 * U) + Q_err) + (UB if bf16 else 2 * U) * y.abs()) * 1.01 + 1e-37
        grad_tol[n][~mask[n]] = 0
    out = dict(loss=loss, loss_tol=loss_tol + 1e-12)
    if grad_loss is not None:
        out.update(grad=grad, grad_tol=grad_tol)
    return out


def embed_backward_reference(grad_out, ids, V, scale, base=None):
    """(dE, its bound) in float64; ``base`` the table's gradient before, if accumulated."""
    bf16 = grad_out.dtype == torch.bfloat16
    N, D = grad_out.shape
    s, mag = torch.zeros((V, D)).double(), torch.zeros((V, D)).double()
    count = torch.zeros(V).double()
    ok = (ids >= 0) & (ids < V)
    at = ids[ok].long()
    s.index_add_(0, at, grad_out[ok].double())
    mag.index_add_(0, at, grad_out[ok].double().abs())
    count.index_add_(0, at, torch.ones(at.shape[0]).double())
    y = s * scale
    tol = (count[:, None] + 4) * U * mag * abs(scale)
    if base is not None:
        y = y + base.double()
        tol = tol + 2 * U * y.abs()
    tol = (tol + (UB if bf16 else U) * y.abs()) * 1.01 + 1e-37
    return y, tol


def check(got, want, tol, what):
    """Every element within its bound; infinities where they are expected."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    diff = (got - want).abs()
    diff[inf] = 0
    bad = ~(diff <= tol)
    bad[inf] = False
    if bad.any():
        i = tuple(int(v) for v in torch.nonzero(bad)[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {i}: got {got[i]}, want {want[i]}, "
                             f"bound {tol[i]}")


def masks(rng, S, V, shares):
    """Truth values [S][V]: state s allows about shares[s % len] of the tokens
    (0: none, 1: all)."""
    share = np.array([shares[s % len(shares)] for s in range(S)])
    return torch.from_numpy(rng.random((S, V)) < share[:, None])
