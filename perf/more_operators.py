"""The operators between a model's last layer and its next token, as they are measured.

Kinds of cases, in the calls that a program makes of them:

  norm      root-mean-square norm of hidden states [N][D] with the residual's
            addition.  ``f8``: the result in 8 bits (e4m3) with a scale for
            every 128 columns, as the 8-bit head product takes it.  ``train``:
            the result in the inputs' type, then both gradients.
  product   the matrix product of 8-bit operands a [M][K] and b [N][K] with a
            scale for every row and 128 k of a and every 128 x 128 of b:
            logits from quantized hidden states and head weights.
  linear    a training step of the same product: activations, weights and the
            output's gradient are quantized, the result and both gradients are
            products of 8-bit operands.
  adjust    logits [B][V] with each sequence's repetition, presence and
            frequency penalties, biases and grammar mask applied.
  tail      the end of a decode step: norm, 8-bit head product, adjustment of
            the logits where they lie.

Sizes: 1 to 8,192 rows, hidden sizes 64 to 8,192, vocabularies of 1,000 to
256,000 tokens, histories of 0 to 16,384 tokens, 0 to 300 biases, bf16 and
fp32, row strides wider than the rows.  Everything is made from the seed:

  hidden    normal, a few columns 20 times as large as the others (as the
            residual stream of a trained model has them).
  history   frequent tokens much more often than rare ones, lengths from
            nothing to the whole buffer, some of it the prompt.
  masks     the allowed tokens of ``S`` automaton states, a state's share of
            the vocabulary drawn from 0.5 % (inside a keyword) to 98 % (inside
            a string); state 0 allows nothing, some rows are dead (state -1).
            ``S`` = 0: no mask.
  biases    moderate ones, bans of -100, unused entries (-1), a token listed
            twice.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
BLOCK = 128                              # columns, or rows and columns, of a scale
TOP = 448.0                              # e4m3's largest
LEAST = 2.0 ** -100                      # a block's largest magnitude counts as this at least
MAX_WORK = 8192 * 4096 * 32000           # rows x columns x k of a drawn product
MAX_LOGITS = 384 * 128256                # rows x tokens of a drawn adjustment
MAX_HIDDEN = 8192 * 4096                 # rows x columns of a drawn norm
EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decoded token through the last norm: latency
        dict(name="norm_f8_1x1024", kind="norm", train=False, f8=True, N=1, D=1024, dtype="bf16", pad=0),
        # a server's batch, eight positions of speculation for each sequence
        dict(name="norm_f8_2304x4096", kind="norm", train=False, f8=True, N=2304, D=4096, dtype="bf16", pad=0),
        # a training batch through the last norm, forward and backward
        dict(name="norm_train_8192x4096", kind="norm", train=True, f8=False, N=8192, D=4096, dtype="bf16", pad=0),
        # a small model in fp32, odd sizes, rows off the usual strides
        dict(name="norm_train_1999x1000_f32", kind="norm", train=True, f8=False, N=1999, D=1000, dtype="f32", pad=9),
        # one token's logits of a small proposer: latency
        dict(name="product_1x1024x32000", kind="product", M=1, K=1024, N=32000, dtype="bf16"),
        # a server's batch through the head of a current model: bound by the weights
        dict(name="product_64x4096x128256", kind="product", M=64, K=4096, N=128256, dtype="bf16"),
        # a small model's training step in fp32, odd sizes
        dict(name="linear_1777x1000x10007_f32", kind="linear", M=1777, K=1000, N=10007, dtype="f32"),
        # the largest: a training step of the head's product
        dict(name="linear_8192x4096x32000", kind="linear", M=8192, K=4096, N=32000, dtype="bf16"),
        # one sequence's logits: latency
        dict(name="adjust_1x32000_f32", kind="adjust", B=1, V=32000, H=512, nb=4, S=16, dtype="f32", pad=0),
        # a server's batch under a grammar
        dict(name="adjust_256x128256", kind="adjust", B=256, V=128256, H=2048, nb=32, S=256, dtype="bf16", pad=0),
        # long histories and long bias lists, odd sizes, a wider buffer, no grammar
        dict(name="adjust_77x50257_f32", kind="adjust", B=77, V=50257, H=16384, nb=300, S=0, dtype="f32", pad=3),
        # the end of a decode step of a server's batch
        dict(name="tail_64x4096x128256", kind="tail", B=64, D=4096, V=128256, H=1024, nb=8, S=64, dtype="bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi, unit):
    """The same, in three of four cases a multiple of ``unit``."""
    n = _spread(rng, lo, hi)
    return n if rng.random() < 0.25 else min(hi, (n + unit - 1) // unit * unit)


def draw(rng):
    kind = rng.choices(["norm", "product", "linear", "adjust", "tail"], [4, 4, 2, 4, 2])[0]
    dtype = rng.choice(["bf16", "bf16", "f32"])
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    if kind == "norm":
        D = _size(rng, 64, 8192, 64)
        N = min(_spread(rng, 1, 8192), MAX_HIDDEN // D // (1 if dtype == "bf16" else 2))
        train = rng.random() < 0.5
        return dict(kind=kind, train=train, f8=not train and rng.random() < 0.7, N=N, D=D, dtype=dtype, pad=pad)
    if kind in ("product", "linear"):
        K, N = _size(rng, 128, 8192, 128), _size(rng, 1000, 128256, 128)
        M = max(1, min(_spread(rng, 1, 8192), MAX_WORK // (K * N) // (1 if kind == "product" else 2)))
        return dict(kind=kind, M=M, K=K, N=N, dtype=dtype)
    V = _size(rng, 1000, 256000, 64)
    S = rng.choice([0, _spread(rng, 4, 256)])
    H, nb = rng.choice([0, _spread(rng, 16, 16384)]), rng.choice([0, _spread(rng, 1, 300)])
    if kind == "adjust":
        B = max(1, min(_spread(rng, 1, 512), MAX_LOGITS // V // (1 if dtype == "bf16" else 2)))
        if not (H or nb or S):
            H = 100
        return dict(kind=kind, B=B, V=V, H=H, nb=nb, S=S, dtype=dtype, pad=pad)
    return dict(kind=kind, B=_spread(rng, 1, 256), D=_size(rng, 128, 4096, 64), V=min(V, 128256), H=max(H, 16), nb=nb, S=S,
                dtype="bf16")


# ------------------------------------------------------------------- inputs

def _up(n):
    return (n + BLOCK - 1) // BLOCK * BLOCK


def _normal(g, n, d, pad, dtype, std=1.0, wide=False):
    """n rows of d normal elements, d + pad apart; ``wide``: a few columns far larger."""
    t = torch.empty((n, d + pad), dtype=dtype, device=DEV)
    size = torch.full((d + pad,), std, device=DEV)
    if wide:
        size[torch.rand(d + pad, generator=g, device=DEV) < 0.004] *= 20.0
    step = max(1, (1 << 26) // (d + pad))
    for i in range(0, n, step):  # made in fp32, a block at a time
        part = t[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * size)
    return t[:, :d]


def _quantized(t, tile):
    """(e4m3 [n][K], scales) of a [n][k] array, K the next multiple of 128 (zeros
    beyond k): by rows, scales [K / 128][n], or by tiles, scales [n / 128][K / 128]."""
    n, k = t.shape
    K, R = _up(k), _up(n) if tile else n
    x = torch.zeros((R, K), device=DEV)
    x[:n, :k] = t
    if tile:
        blocks = x.view(R // BLOCK, BLOCK, K // BLOCK, BLOCK)
        scales = blocks.abs().amax((1, 3)).clamp(min=LEAST) / TOP
        q = blocks / scales[:, None, :, None]
        return q.view(R, K)[:n].to(torch.float8_e4m3fn), scales
    blocks = x.view(n, K // BLOCK, BLOCK)
    scales = blocks.abs().amax(2).clamp(min=LEAST) / TOP
    return (blocks / scales[:, :, None]).view(n, K).to(torch.float8_e4m3fn), scales.t().contiguous()


def _mask(g, S, V, B):
    """allow [S][ceil(V/32)] int32 and states [B] int32."""
    lo, hi = math.log(0.005), math.log(0.98)
    share = torch.exp(lo + (hi - lo) * torch.rand(S, generator=g, device=DEV) ** 0.5)
    words = (V + 31) // 32
    allow = torch.empty((S, words), dtype=torch.int32, device=DEV)
    for s in range(S):
        bits = torch.rand(words * 32, generator=g, device=DEV) < share[s]
        bits[V:] = False
        if s == 0:
            bits[:] = False
        packed = (bits.view(words, 32).to(torch.int64) << torch.arange(32, device=DEV)).sum(1)
        allow[s] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
    states = torch.randint(min(1, S - 1), S, (B,), generator=g, device=DEV, dtype=torch.int32)
    if B > 8:  # a row that the mask leaves empty, and a dead one
        at = torch.randperm(B, generator=g, device=DEV)
        states[at[0]] = 0
        states[at[1]] = -1
    return allow, states


def _requests(g, case, state):
    """What the sequences of a batch ask for: histories, penalties, biases, masks."""
    B, V, H, nb, S = (case[k] for k in ("B", "V", "H", "nb", "S"))
    u = lambda *shape: torch.rand(shape, generator=g, device=DEV)  # noqa: E731
    zipf = lambda *shape: (V ** u(*shape) - 1).long().clamp(0, V - 1).to(torch.int32)  # noqa: E731
    for k in ("history", "lengths", "prompts", "repetition", "presence", "frequency", "bias_ids", "bias", "allow", "states"):
        state[k] = None
    if H:
        state["history"] = zipf(B, H)
        lengths = (u(B) * (H + 1)).long().clamp(max=H)
        lengths[0] = H
        if B > 4:
            lengths[1] = 0
        state["lengths"] = lengths.to(torch.int32)
        state["prompts"] = (u(B) * lengths).to(torch.int32)
        state["repetition"] = 1.0 + 0.3 * u(B)
        state["presence"] = 1.5 * u(B) - 0.25
        state["frequency"] = 0.5 * u(B)
    if nb:
        ids = torch.randint(0, V, (B, nb), generator=g, device=DEV, dtype=torch.int32)
        bias = torch.randn((B, nb), generator=g, device=DEV) * 3.0
        bias = torch.where(u(B, nb) < 0.2, -100.0, bias)
        ids = torch.where(u(B, nb) < 0.1, -1, ids)
        if nb > 2:
            ids[:, nb - 1] = ids[:, 0]
        state["bias_ids"], state["bias"] = ids.contiguous(), bias
    if S:
        state["allow"], state["states"] = _mask(g, S, V, B)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 31)
    s = dict(case)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    if kind == "norm":
        N, D, pad = case["N"], case["D"], case["pad"]
        s["x"] = _normal(g, N, D, pad, dtype)
        s["residual"] = _normal(g, N, D, pad, dtype, 2.0, wide=True)
        s["weight"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
        if case["train"]:
            s["grad_out"] = _normal(g, N, D, 0, dtype, 1.0 / N)
            s["grad_total"] = _normal(g, N, D, 0, dtype, 1.0 / N)
    elif kind == "product":
        M, K, N = case["M"], case["K"], case["N"]
        s["a"], s["sa"] = _quantized(_normal(g, M, K, 0, torch.float32, wide=True), False)
        s["b"], s["sb"] = _quantized(_normal(g, N, K, 0, torch.bfloat16, 1.0 / math.sqrt(K)), True)
    elif kind == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = _normal(g, M, K, 0, dtype, wide=True)
        s["weight"] = _normal(g, N, K, 0, dtype, 1.0 / math.sqrt(K))
        s["grad_out"] = _normal(g, M, N, 0, dtype, 1.0 / M)
    else:
        _requests(g, case, s)
        if kind == "adjust":
            s["logits"] = _normal(g, case["B"], case["V"], case["pad"], dtype, 3.0)
        else:
            B, D, V = case["B"], case["D"], case["V"]
            s["x"] = _normal(g, B, D, 0, dtype)
            s["residual"] = _normal(g, B, D, 0, dtype, 2.0, wide=True)
            s["weight"] = (1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(dtype)
            s["head"], s["head_scales"] = _quantized(_normal(g, V, D, 0, torch.bfloat16, 3.0 / math.sqrt(D)), True)
    return s


# ---------------------------------------------------------------- plain forms

def _norm(x, residual, weight):
    """(h in the inputs' type, y and 1 / rms in fp32)."""
    h = (x.float() + residual.float()).to(x.dtype)
    hf = h.float()
    r = 1.0 / torch.sqrt((hf * hf).mean(1, keepdim=True) + EPS)
    return h, hf * r * weight.float(), r


def _blocks(x, tile):
    """A [n][k] array, zeros up to whole blocks: by rows [n][kb][128], or by tiles
    [nb][128][kb][128]."""
    n, k = x.shape
    x = torch.nn.functional.pad(x, (0, _up(k) - k, 0, _up(n) - n if tile else 0))
    if tile:
        return x.view(x.shape[0] // BLOCK, BLOCK, x.shape[1] // BLOCK, BLOCK)
    return x.view(n, x.shape[1] // BLOCK, BLOCK)


def _quantize(x, tile=False):
    """(e4m3 blocks, their scales with ones for the block's dimensions)."""
    b = _blocks(x, tile)
    largest = b.abs().amax((1, 3) if tile else 2, keepdim=True).clamp(min=LEAST)
    scales = largest / torch.full_like(largest, TOP)  # (a number there becomes a product with its reciprocal)
    return (b / scales).to(torch.float8_e4m3fn), scales


def _values(q, scales, n):
    """What quantized blocks stand for, [n][K] in fp32."""
    v = q.float() * scales
    return v.reshape(-1, v.shape[-1] * v.shape[-2])[:n] if v.dim() == 3 else v.reshape(v.shape[0] * BLOCK, -1)[:n]


def _plain_norm(s):
    h, y, r = _norm(s["x"], s["residual"], s["weight"])
    if s["f8"]:
        q, scales = _quantize(y)
        return q.view(s["N"], -1), scales[:, :, 0].t().contiguous(), h
    out = y.to(h.dtype)
    if not s["train"]:
        return out, h
    hf, g = h.float(), s["grad_out"].float()
    gw = g * s["weight"].float()
    dx = r * gw - hf * (r * r * r * (gw * hf).mean(1, keepdim=True)) + s["grad_total"].float()
    dw = (g * hf * r).sum(0)
    return out, h, dx.to(h.dtype), dw.to(h.dtype)


def _plain_product(s):
    M, N, K = s["M"], s["N"], s["a"].shape[1]
    a = (s["a"].float().view(M, -1, BLOCK) * s["sa"].t()[:, :, None]).view(M, K)
    sb = s["sb"].repeat_interleave(BLOCK, 0)[:N]
    b = (s["b"].float().view(N, -1, BLOCK) * sb[:, :, None]).view(N, K)
    return (a @ b.t()).to(DTYPES[s["dtype"]])


def _plain_linear(s):
    M, K, N = s["M"], s["K"], s["N"]
    x, w, g = s["x"].float(), s["weight"].float(), s["grad_out"].float()
    wv = _values(*_quantize(w, tile=True), N)[:, :K]
    out = _values(*_quantize(x), M)[:, :K] @ wv.t()
    gx = _values(*_quantize(g), M)[:, :N] @ wv
    # along the rows, for the weight's gradient
    gw = _values(*_quantize(g.t()), N) @ _values(*_quantize(x.t()), K).t()
    return out.to(s["x"].dtype), gx.to(s["x"].dtype), gw.to(s["x"].dtype)


def _adjusted(z, s):
    """fp32 logits with the requests applied."""
    B, V = z.shape
    if s["history"] is not None:
        H = s["history"].shape[1]
        at = torch.arange(H, device=z.device)[None, :]
        live = at < s["lengths"][:, None]
        made = live & (at >= s["prompts"][:, None])
        ids = s["history"].long()
        seen = torch.zeros((B, V), device=z.device).scatter_add_(1, ids, live.float()) > 0
        count = torch.zeros((B, V), device=z.device).scatter_add_(1, ids, made.float())
        rho = s["repetition"][:, None]
        z = torch.where(seen, torch.where(z > 0, z / rho, z * rho), z)
        z = z - count * s["frequency"][:, None] - torch.where(count > 0, s["presence"][:, None], 0.0)
    if s["bias_ids"] is not None:
        ids = s["bias_ids"].long()
        inside = (ids >= 0) & (ids < V)
        z = z + torch.zeros((B, V), device=z.device).scatter_add_(1, ids.clamp(0, V - 1), torch.where(inside, s["bias"], 0.0))
    if s["allow"] is not None:
        S = s["allow"].shape[0]
        live = (s["states"] >= 0) & (s["states"] < S)
        words = s["allow"][s["states"].long().clamp(0, S - 1)].repeat_interleave(32, dim=1)[:, :V]
        may = ((words >> (torch.arange(V, device=z.device) % 32).to(torch.int32)) & 1).bool() & live[:, None]
        z = torch.where(may, z, -math.inf)
    return z


def _plain_adjust(s):
    return _adjusted(s["logits"].float(), s).to(s["logits"].dtype)


def _plain_tail(s):
    B, V = s["B"], s["V"]
    h, y, _ = _norm(s["x"], s["residual"], s["weight"])
    a = _values(*_quantize(y), B)
    sb = s["head_scales"].repeat_interleave(BLOCK, 0)[:V]
    b = (s["head"].float().view(V, -1, BLOCK) * sb[:, :, None]).view(V, -1)
    z = (a @ b.t()).to(h.dtype)               # the logits are kept in the inputs' type
    return h, _adjusted(z.float(), s).to(h.dtype)


def _own(s):
    import paper_2403_06988_amd as dv

    kind = s["kind"]
    if kind == "norm":
        if s["f8"]:
            return dv.rms_norm_f8(s["x"], s["weight"], EPS, residual=s["residual"])
        out, total, rstd = dv.rms_norm(s["x"], s["weight"], EPS, residual=s["residual"], want_rstd=s["train"])
        if not s["train"]:
            return out, total
        return out, total, *dv.rms_norm_backward(s["grad_out"], total, s["weight"], rstd, grad_total=s["grad_total"])
    if kind == "product":
        return dv.product_f8(s["a"], s["sa"], s["b"], s["sb"], tile=BLOCK, dtype=DTYPES[s["dtype"]])
    if kind == "linear":
        dtype, K, N = s["x"].dtype, s["K"], s["N"]
        xq, xs, xt, xts = dv.quantize_f8(s["x"], want_columns=True)
        wq, ws, wt, wts = dv.quantize_f8(s["weight"], tile=BLOCK, want_columns=True)
        out = dv.product_f8(xq, xs, wq, ws, tile=BLOCK, dtype=dtype)
        gq, gs, gt, gts = dv.quantize_f8(s["grad_out"], want_columns=True)
        gx = dv.product_f8(gq, gs, wt, wts, tile=BLOCK, dtype=dtype)
        gw = dv.product_f8(gt, gts, xt, xts, tile=1, dtype=dtype)
        return out, gx, gw
    how = dict(history=s["history"], lengths=s["lengths"], prompt_lengths=s["prompts"], repetition=s["repetition"],
               presence=s["presence"], frequency=s["frequency"], bias_ids=s["bias_ids"], bias=s["bias"],
               allow=s["allow"], states=s["states"])
    if kind == "adjust":
        return dv.adjust_logits(s["logits"], **how)
    q, scales, total = dv.rms_norm_f8(s["x"], s["weight"], EPS, residual=s["residual"])
    z = dv.product_f8(q, scales, s["head"], s["head_scales"], tile=BLOCK, dtype=total.dtype)
    return total, dv.adjust_logits(z, out=z, **how)


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "product": _plain_product, "linear": _plain_linear, "adjust": _plain_adjust,
            "tail": _plain_tail}[state["kind"]](state)


def _request_bytes(c):
    b = 0
    if c["H"]:
        b += c["B"] * (4 * c["H"] // 2 + 20)          # half the history buffers are filled
    if c["S"]:
        b += 4 * c["B"] + min(c["B"], c["S"]) * ((c["V"] + 31) // 32) * 4
    return b + 8 * c["B"] * c["nb"]


def work(case):
    """What one pass cannot do without: every input read once, every output
    written once, the products' multiplications and additions."""
    c, kind, elt = case, case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "norm":
        N, D = c["N"], c["D"]
        b = (3 * N * D + D) * elt + (N * _up(D) * (1 + 4 / BLOCK) if c["f8"] else N * D * elt)
        if c["train"]:
            b += (4 * N * D + 2 * D) * elt + 8 * N
        return {"bytes": b, "flops": N * D * (16 if c["train"] else 6)}
    if kind == "product":
        M, K, N = c["M"], _up(c["K"]), c["N"]
        b = (M + N) * K + 4 * (M + _up(N) // BLOCK) * (K // BLOCK) + M * N * elt
        return {"bytes": b, "flops": 2 * M * N * c["K"]}
    if kind == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        return {"bytes": 2 * (M * K + N * K + M * N) * elt, "flops": 6 * M * N * K}
    if kind == "adjust":
        return {"bytes": 2 * c["B"] * c["V"] * elt + _request_bytes(c), "flops": c["B"] * c["V"]}
    B, D, V = c["B"], _up(c["D"]), c["V"]
    return {"bytes": 3 * B * c["D"] * elt + V * D + B * V * elt + _request_bytes(c), "flops": 2 * B * V * c["D"]}


# ------------------------------------------------------------- 64-bit results

def _round8(v):
    """The nearest e4m3 value of each element (ties to the even one)."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(v / step) * step


def _stands_for(v, rows, cols):
    """v in 64 bits, quantized in blocks of ``rows`` x ``cols``: what it then stands for."""
    out = torch.empty_like(v)
    cut = max(1, (1 << 26) // max(1, v.shape[1] * rows)) * rows
    for i in range(0, v.shape[0], cut):
        part = v[i:i + cut]
        n, k = part.shape
        p = torch.zeros((-(-n // rows) * rows, -(-k // cols) * cols), dtype=v.dtype, device=v.device)
        p[:n, :k] = part
        largest = p.unfold(0, rows, rows).unfold(1, cols, cols).abs().amax((2, 3))
        # a scale and a quotient are numbers of 32 bits: with 448 = 7 * 64, many quotients of bf16
        # values lie on the border between two e4m3 values, or next to it
        scale = (torch.clamp(largest, min=LEAST) / TOP).float().double()
        scale = scale.repeat_interleave(rows, 0).repeat_interleave(cols, 1)
        out[i:i + cut] = (_round8((p / scale).float().double()) * scale)[:n, :k]
    return out


def _exact_norm(s):
    x, res, w = s["x"].double(), s["residual"].double(), s["weight"].double()
    total = x + res
    h = total.to(s["x"].dtype).double()               # what the norm is taken of, as it is kept
    mean = h.pow(2).sum(1, keepdim=True) / h.shape[1]
    unit = h * torch.rsqrt(mean + EPS)
    return total, h, mean, unit, unit * w


def _exact_adjust(z, s):
    B, V = z.shape
    for b in range(B):
        row = z[b]
        if s["history"] is not None:
            n, p = int(s["lengths"][b]), int(s["prompts"][b])
            ids = s["history"][b, :n].long()
            seen = torch.bincount(ids, minlength=V)
            made = torch.bincount(ids[p:], minlength=V).double()
            rho = s["repetition"][b].double()
            k = torch.nonzero(seen)[:, 0]
            row[k] = torch.where(row[k] > 0, row[k] / rho, row[k] * rho)
            row -= made * s["frequency"][b].double()
            row[made > 0] -= s["presence"][b].double()
        if s["bias_ids"] is not None:
            ids = s["bias_ids"][b].long()
            keep = (ids >= 0) & (ids < V)
            row.index_add_(0, ids[keep], s["bias"][b][keep].double())
        if s["allow"] is not None:
            state = int(s["states"][b])
            if 0 <= state < s["allow"].shape[0]:
                word = s["allow"][state].long() & 0xFFFFFFFF
                bit = torch.arange(V, device=z.device)
                row[(word[bit // 32] >> (bit % 32)) % 2 == 0] = -math.inf
            else:
                row.fill_(-math.inf)
    return z


def exact(case, seed):
    """The definitions evaluated in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        total, h, mean, unit, y = _exact_norm(s)
        if case["f8"]:
            N, D = y.shape
            p = torch.zeros((N, _up(D)), dtype=torch.float64, device=DEV)
            p[:, :D] = y
            scale = p.unfold(1, BLOCK, BLOCK).abs().amax(2).clamp(min=LEAST) / TOP
            return p / scale.repeat_interleave(BLOCK, 1), scale.t(), total
        if not case["train"]:
            return y, total
        g, w = s["grad_out"].double(), s["weight"].double()
        r = torch.rsqrt(mean + EPS)
        along = (g * w * unit).sum(1, keepdim=True) / h.shape[1]
        return y, total, r * (g * w - unit * along) + s["grad_total"].double(), (g * unit).sum(0)
    if kind == "product":
        a = s["a"].double() * s["sa"].double().repeat_interleave(BLOCK, 0).t()
        n = case["N"]
        sb = s["sb"].double().repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)
        return torch.matmul(a, (s["b"].double() * sb).transpose(0, 1))
    if kind == "linear":
        x, w, g = s["x"].double(), s["weight"].double(), s["grad_out"].double()
        wv = _stands_for(w, BLOCK, BLOCK)
        out = torch.matmul(_stands_for(x, 1, BLOCK), wv.transpose(0, 1))
        gx = torch.matmul(_stands_for(g, 1, BLOCK), wv)
        gw = torch.matmul(_stands_for(g, BLOCK, 1).transpose(0, 1), _stands_for(x, BLOCK, 1))
        return out, gx, gw
    if kind == "adjust":
        return _exact_adjust(s["logits"].double(), s)
    total, _, _, _, y = _exact_norm(s)
    V, D = case["V"], case["D"]
    sb = s["head_scales"].double().repeat_interleave(BLOCK, 0)[:V].repeat_interleave(BLOCK, 1)
    z = torch.matmul(_stands_for(y, 1, BLOCK), (s["head"].double() * sb)[:, :D].transpose(0, 1))
    return total, _exact_adjust(z.to(DTYPES[case["dtype"]]).double(), s)   # the logits as they are kept
