"""The training operators at the vocabulary end of a model, as they are measured.

Three operators, in the calls that a program makes of them:

  head     softmax cross entropy over the tokens that each row's automaton
           state allows, from hidden states x [N][D] and head weights w [V][D]:
           the loss alone (``train`` false), or the loss and then both
           gradients.
  distill  the divergence of a model's logits [N][V] from a teacher's top K
           logits, over the allowed tokens: the loss alone, or the loss with
           the gradient of the logits.
  embed    rows of a table [V][D] looked up by token and scaled: the lookup
           alone, or the lookup and then the table's gradient.

Sizes: 1 to 8,192 rows, hidden sizes 64 to 4,096, vocabularies of 1,000 to
256,000 tokens, 4 to 256 teacher logits, bf16 and fp32, row strides wider than
the rows.  Everything is made from the seed:

  masks    the allowed tokens of ``S`` automaton states, a state's share of the
           vocabulary drawn from 0.5 % (inside a keyword) to 98 % (inside a
           string); state 0 allows nothing, and some rows are dead (state -1).
           ``S`` = 0: no mask.
  targets  an allowed token of the row's state, for a twentieth of the rows -1
           (padding) or any token, allowed or not.
  hidden   normal, plus a share of the target's weight row: from rows that know
           nothing of their target to rows that are sure of it.
  teacher  descending logits, the ids near the top of the student's own
           order for some and anywhere for the others.
  tokens   frequent ones much more often than rare ones, a hundredth padding
           (-1).
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
MAX_WORK = 8192 * 4096 * 128256       # rows x hidden x tokens of a drawn head case
MAX_LOGITS = 2048 * 128256            # rows x tokens of a drawn distillation
MAX_TABLE = 128256 * 4096             # tokens x hidden of a drawn table
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the token just generated scored under its constraint: latency
        dict(name="head_score_1x1024x32000", kind="head", train=False, N=1, D=1024, V=32000, S=64, dtype="bf16", pad=0),
        # a batch of an evaluation, no constraint
        dict(name="head_eval_512x2048x128256", kind="head", train=False, N=512, D=2048, V=128256, S=0, dtype="bf16", pad=0),
        # a small proposer's training step: odd sizes, rows off the usual strides, a constraint
        dict(name="head_train_1999x1000x32003", kind="head", train=True, N=1999, D=1000, V=32003, S=92, dtype="bf16", pad=9),
        # the largest: a batch of tokens through the head of a current model
        dict(name="head_train_8192x4096x128256", kind="head", train=True, N=8192, D=4096, V=128256, S=256, dtype="bf16", pad=0),
        # a small model trained in fp32
        dict(name="head_train_1024x512x32000_f32", kind="head", train=True, N=1024, D=512, V=32000, S=0, dtype="f32", pad=0),
        # a few rows compared with their teacher while serving
        dict(name="distill_eval_8x32000_f32", kind="distill", train=False, N=8, V=32000, K=16, S=16, dtype="f32", pad=0, inv_t=1.0),
        # a distillation step on a current tokenizer, under a constraint
        dict(name="distill_train_2048x128256", kind="distill", train=True, N=2048, V=128256, K=64, S=256, dtype="bf16", pad=0, inv_t=1.0),
        # odd sizes, fp32 logits in a wider buffer, a softened teacher
        dict(name="distill_train_333x50257_f32", kind="distill", train=True, N=333, V=50257, K=20, S=0, dtype="f32", pad=3, inv_t=0.5),
        # few rows of a large vocabulary
        dict(name="distill_train_40x256000", kind="distill", train=True, N=40, V=256000, K=100, S=64, dtype="bf16", pad=0, inv_t=1.0),
        # the tokens of one decode step of a server's batch
        dict(name="embed_64x4096x128256", kind="embed", train=False, N=64, D=4096, V=128256, dtype="bf16", scale=1.0),
        # a training batch of a middling model: lookup and the table's gradient
        dict(name="embed_train_8192x2048x128256", kind="embed", train=True, N=8192, D=2048, V=128256, dtype="bf16", scale=45.25),
        # a small model in fp32, odd sizes
        dict(name="embed_train_5001x777x32003_f32", kind="embed", train=True, N=5001, D=777, V=32003, dtype="f32", scale=1.0),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _hidden(rng):
    D = _spread(rng, 64, 4096)
    r = rng.random()
    return D if r < 0.25 else min(4096, (D + 63) // 64 * 64)


def draw(rng):
    kind = rng.choices(["head", "distill", "embed"], [5, 4, 3])[0]
    V = _spread(rng, 1000, 256000)
    if rng.random() < 0.5:
        V = (V + 63) // 64 * 64
    dtype = rng.choice(["bf16", "bf16", "f32"])
    N = _spread(rng, 1, 8192)
    S = rng.choice([0, _spread(rng, 4, 256)])
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    if kind == "head":
        D = _hidden(rng)
        N = max(1, min(N, MAX_WORK // (D * V)))
        return dict(kind=kind, train=rng.random() < 0.6, N=N, D=D, V=V, S=S, dtype=dtype, pad=pad)
    if kind == "distill":
        N = max(1, min(N, MAX_LOGITS // V // (1 if dtype == "bf16" else 2)))
        return dict(kind=kind, train=rng.random() < 0.7, N=N, V=V, K=_spread(rng, 4, 256), S=S, dtype=dtype, pad=pad,
                    inv_t=rng.choice([0.5, 1.0, 1.25]))
    D = _hidden(rng)
    D = max(64, min(D, MAX_TABLE // V))
    return dict(kind=kind, train=rng.random() < 0.6, N=N, D=D, V=V, dtype=dtype, scale=rng.choice([1.0, math.sqrt(D)]))


# ------------------------------------------------------------------- inputs

def _rows(g, n, d, pad, dtype, std=1.0):
    """n rows of d normal elements, d + pad apart."""
    t = torch.empty((n, d + pad), dtype=dtype, device=DEV)
    step = max(1, (1 << 26) // (d + pad))
    for i in range(0, n, step):  # made in fp32, a block at a time
        part = t[i:i + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std)
    return t[:, :d]


def _masks(g, case):
    """(allow [S][ceil(V/32)] int32, the same as truth values [S][V], states [N])."""
    S, V, N = case["S"], case["V"], case["N"]
    lo, hi = math.log(0.005), math.log(0.98)
    share = torch.exp(lo + (hi - lo) * torch.rand(S, generator=g, device=DEV) ** 0.5)
    may = torch.rand((S, V), generator=g, device=DEV) < share[:, None]
    may[:, 0] = True
    may[0] = False
    words = (V + 31) // 32
    bits = torch.zeros((S, words * 32), dtype=torch.int64, device=DEV)
    bits[:, :V] = may
    packed = (bits.view(S, words, 32) << torch.arange(32, device=DEV)).sum(-1)
    allow = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
    states = torch.randint(1, S, (N,), generator=g, device=DEV, dtype=torch.int32)
    u = torch.rand(N, generator=g, device=DEV)
    if N > 8:  # rows that the mask leaves empty, and dead ones
        states = torch.where(u < 0.01, torch.zeros_like(states), torch.where(u > 0.99, torch.full_like(states, -1), states))
    return allow, may, states


def _allowed_token(g, may, states, N, V):
    """A token that each row's state allows (0 where it allows none)."""
    u = torch.rand(N, generator=g, device=DEV)
    if may is None:
        return (u * V).long().clamp(max=V - 1)
    count = may.sum(1)
    order = torch.argsort(may.int(), dim=1, descending=True, stable=True)   # a state's allowed tokens first
    s = states.long().clamp(min=0)
    k = (u * count[s]).long()
    return order[s, torch.minimum(k, (count[s] - 1).clamp(min=0))]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1_000_003 + 29)
    state = dict(case)
    dtype = DTYPES[case["dtype"]]
    N, V = case["N"], case["V"]
    if case["kind"] == "embed":
        state["weight"] = _rows(g, V, case["D"], 0, dtype)
        u = torch.rand(N, generator=g, device=DEV)
        ids = (V ** u - 1).long().clamp(0, V - 1)                  # token i about as often as 1 / (i + 1)
        if N > 8:
            ids = torch.where(torch.rand(N, generator=g, device=DEV) < 0.01, -1, ids)
        state["ids"] = ids.to(torch.int32)
        if case["train"]:
            state["grad_out"] = _rows(g, N, case["D"], 0, dtype, 1.0 / N)
        return state
    allow = may = states = None
    if case["S"]:
        allow, may, states = _masks(g, case)
    state["allow"], state["states"] = allow, states
    if case["train"]:
        state["grad_loss"] = (0.5 + torch.rand(N, generator=g, device=DEV)) / N   # weights of a mean
    target = _allowed_token(g, may, states, N, V)
    if case["kind"] == "head":
        D = case["D"]
        state["weight"] = _rows(g, V, D, case["pad"], dtype, 3.0 / math.sqrt(D))
        x = torch.empty((N, D + case["pad"]), dtype=dtype, device=DEV)[:, :D]
        sure = 4.0 * torch.rand((N, 1), generator=g, device=DEV) / 3.0
        x.copy_(torch.randn((N, D), generator=g, device=DEV) + sure * state["weight"][target].float())
        state["x"] = x
        if N > 8:
            u = torch.rand(N, generator=g, device=DEV)
            anywhere = torch.randint(0, V, (N,), generator=g, device=DEV)
            target = torch.where(u < 0.03, -1, torch.where(u > 0.98, anywhere, target))
        state["targets"] = target.to(torch.int32)
        return state
    K = case["K"]
    state["logits"] = _rows(g, N, V, case["pad"], dtype, 3.0)
    order = torch.empty((N, K), dtype=torch.int64, device=DEV)
    for i in range(0, N, 256):
        order[i:i + 256] = state["logits"][i:i + 256].float().topk(K, dim=1).indices
    anywhere = torch.randint(0, V, (N, K), generator=g, device=DEV)
    ids = torch.where(torch.rand((N, K), generator=g, device=DEV) < 0.6, order, anywhere)
    ids[:, 0] = target
    state["teacher_ids"] = ids.to(torch.int32)
    top = torch.randn((N, K), generator=g, device=DEV) * 2.5 + 8.0
    state["teacher_logits"] = top.sort(1, descending=True).values
    return state


# ---------------------------------------------------------------- plain forms

def _bits(allow, states, V):
    """Which tokens each row allows, [N][V]."""
    live = (states >= 0) & (states < allow.shape[0])
    rows = states.long().clamp(0, allow.shape[0] - 1)
    few = rows.shape[0] < allow.shape[0]
    words = (allow[rows] if few else allow).repeat_interleave(32, dim=1)[:, :V]
    may = ((words >> (torch.arange(V, device=allow.device) % 32).to(torch.int32)) & 1).bool()
    return (may if few else may[rows]) & live[:, None]


def _plain_softmax(z, may):
    """(exp(z - max), its sum, the maximum) over the allowed tokens of each row;
    a row without any has sum 0."""
    if may is not None:
        z = z.masked_fill(~may, -math.inf)
    m = z.max(1, keepdim=True).values
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    e = torch.exp(z - m)
    return e, e.sum(1, keepdim=True), m


def _plain_head(s):
    V, dtype = s["V"], s["weight"].dtype
    x, w, t = s["x"].float(), s["weight"].float(), s["targets"].long()[:, None]
    z = x @ w.t()
    may = None if s["allow"] is None else _bits(s["allow"], s["states"], V)
    e, total, m = _plain_softmax(z, may)
    lse = (m + torch.log(total))[:, 0]
    part = (t >= 0) & (t < V)
    t = t.clamp(0, V - 1)
    if may is not None:
        part = part & may.gather(1, t)
    loss = torch.where(part[:, 0], lse - z.gather(1, t)[:, 0], 0.0)
    if not s["train"]:
        return loss, lse
    g = torch.where(part, s["grad_loss"][:, None], 0.0)
    p = e * torch.where(part, g / total, 0.0)
    p.scatter_add_(1, t, -g)
    return loss, lse, (p @ w).to(dtype), (p.t() @ x).to(dtype)


def _plain_distill(s):
    V, c = s["V"], s["inv_t"]
    ids, top = s["teacher_ids"].long(), s["teacher_logits"].float() * c
    may = None if s["allow"] is None else _bits(s["allow"], s["states"], V)
    e, total, m = _plain_softmax(s["logits"].float() * c, may)
    listed_ = (ids >= 0) & (ids < V)
    ids = ids.clamp(0, V - 1)
    if may is not None:
        listed_ = listed_ & may.gather(1, ids)
    q, qs, qm = _plain_softmax(top, listed_)
    part = (qs > 0) & (total > 0)
    logq = top - qm - torch.log(qs)
    q = torch.where(part, q / qs, 0.0)
    logp = (s["logits"].gather(1, ids).float() * c - m) - torch.log(total)
    loss = torch.where(q > 0, q * (logq - logp), 0.0).sum(1)
    if not s["train"]:
        return loss
    g = torch.where(part, s["grad_loss"][:, None] * c, 0.0)
    d = e * torch.where(part, g / total, 0.0)
    d.scatter_add_(1, ids, -g * q)
    return loss, d.to(s["logits"].dtype)


def _plain_embed(s):
    w, dtype = s["weight"], s["weight"].dtype
    ids = s["ids"].long()
    inside = ((ids >= 0) & (ids < s["V"]))[:, None]
    at = ids.clamp(0, s["V"] - 1)
    out = torch.where(inside, w[at].float() * s["scale"], 0.0).to(dtype)
    if not s["train"]:
        return out
    grad = torch.zeros(w.shape, dtype=torch.float32, device=w.device)
    grad.index_add_(0, at, torch.where(inside, s["grad_out"].float() * s["scale"], 0.0))
    return out, grad.to(dtype)


def _own(s):
    import paper_2403_06988_amd as dv

    if s["kind"] == "head":
        mask = dict(allow=s["allow"], states=s["states"])
        loss, lse = dv.head_loss(s["x"], s["weight"], s["targets"], **mask)
        if not s["train"]:
            return loss, lse
        gx, gw = dv.head_loss_backward(s["x"], s["weight"], s["targets"], lse, s["grad_loss"], **mask)
        return loss, lse, gx, gw
    if s["kind"] == "distill":
        args = (s["logits"], s["teacher_ids"], s["teacher_logits"])
        how = dict(inv_temperature=s["inv_t"], allow=s["allow"], states=s["states"])
        if not s["train"]:
            return dv.distill_loss(*args, **how)
        return dv.distill_loss_backward(*args, s["grad_loss"], **how)
    out = dv.embed(s["weight"], s["ids"], scale=s["scale"])
    if not s["train"]:
        return out
    return out, dv.embed_backward(s["grad_out"], s["ids"], s["V"], scale=s["scale"])


def run(state):
    if own:
        return _own(state)
    return {"head": _plain_head, "distill": _plain_distill, "embed": _plain_embed}[state["kind"]](state)


def work(case):
    """What one pass cannot do without: every input read once, every output
    written once, the products' multiplications and additions."""
    N, V, elt = case["N"], case["V"], 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "embed":
        b = 2 * N * case["D"] * elt + 4 * N
        if case["train"]:
            b += (N + V) * case["D"] * elt
        return {"bytes": b, "flops": N * case["D"] * (2 if case["train"] else 1)}
    S = case["S"]
    mask = 4 * N + min(N, S) * ((V + 31) // 32) * 4 if S else 0
    if case["kind"] == "distill":
        b = N * V * elt * (2 if case["train"] else 1) + 8 * N * case["K"] + 8 * N + mask
        return {"bytes": b, "flops": N * V * (6 if case["train"] else 4)}
    D = case["D"]
    b = (N + V) * D * elt * (2 if case["train"] else 1) + 12 * N + mask + (4 * N if case["train"] else 0)
    return {"bytes": b, "flops": N * D * V * (6 if case["train"] else 2)}


# ------------------------------------------------------------- 64-bit results

def exact(case, seed):
    """The definitions evaluated in 64 bits, a block of rows at a time."""
    s = prepare(case, seed)
    V, N = case["V"], case["N"]
    f64 = dict(dtype=torch.float64, device=DEV)
    if case["kind"] == "embed":
        ok = torch.nonzero((s["ids"] >= 0) & (s["ids"] < V))[:, 0]
        at = s["ids"][ok].long()
        out = torch.zeros((N, case["D"]), **f64)
        out[ok] = s["weight"][at].double() * case["scale"]
        if not case["train"]:
            return out
        grad = torch.zeros((V, case["D"]), **f64)
        grad.index_add_(0, at, s["grad_out"][ok].double())
        return out, grad * case["scale"]
    bit = torch.arange(V, device=DEV)

    def admitted(i, j):
        if s["allow"] is None:
            return torch.ones((j - i, V), dtype=torch.bool, device=DEV)
        st = s["states"][i:j].long()
        ok = torch.zeros((j - i, V), dtype=torch.bool, device=DEV)
        for r in range(j - i):
            if 0 <= int(st[r]) < case["S"]:
                word = s["allow"][int(st[r])].long() & 0xFFFFFFFF
                ok[r] = (word[bit // 32] >> (bit % 32)) % 2 == 1
        return ok

    step = max(1, (1 << 27) // V)
    if case["kind"] == "head":
        x, w, target = s["x"].double(), s["weight"].double(), s["targets"].tolist()
        loss, lse = torch.zeros(N, **f64), torch.zeros(N, **f64)
        gx = torch.zeros(x.shape, **f64) if case["train"] else None
        gw = torch.zeros(w.shape, **f64) if case["train"] else None
        for i in range(0, N, step):
            j = min(N, i + step)
            ok = admitted(i, j)
            z = torch.matmul(x[i:j], w.transpose(0, 1))
            z[~ok] = -math.inf
            lse[i:j] = torch.logsumexp(z, 1)
            rows = [r for r in range(j - i) if 0 <= target[i + r] < V]
            t = torch.tensor([target[i + r] for r in rows], dtype=torch.int64, device=DEV)
            r = torch.tensor(rows, dtype=torch.int64, device=DEV)
            keep = ok[r, t]
            r, t = r[keep], t[keep]
            loss[i + r] = lse[i + r] - z[r, t]
            if case["train"]:
                d = torch.zeros_like(z)
                d[r] = torch.exp(z[r] - lse[i + r][:, None])
                d[r, t] -= 1.0
                d *= s["grad_loss"][i:j].double()[:, None]
                gx[i:j] = torch.matmul(d, w)
                gw += torch.matmul(d.transpose(0, 1).contiguous(), x[i:j])
        return (loss, lse, gx, gw) if case["train"] else (loss, lse)
    loss = torch.zeros(N, **f64)
    grad = torch.zeros((N, V), **f64) if case["train"] else None
    for i in range(0, N, step):
        j = min(N, i + step)
        ok = admitted(i, j)
        z = s["logits"][i:j].double() * case["inv_t"]
        z[~ok] = -math.inf
        logp = z - torch.logsumexp(z, 1, keepdim=True)
        ids, top = s["teacher_ids"][i:j].long(), s["teacher_logits"][i:j].double() * case["inv_t"]
        good = ok.gather(1, ids)
        top = torch.where(good, top, torch.full_like(top, -math.inf))
        rows = good.any(1)
        logq = (top - torch.logsumexp(top, 1, keepdim=True))[rows]
        q = torch.exp(logq)
        at = ids[rows]
        diff = torch.where(q > 0, logq - logp[rows].gather(1, at), torch.zeros_like(q))
        loss[i:j][rows] = (q * diff).sum(1)
        if case["train"]:
            d = torch.exp(logp[rows])
            d.scatter_add_(1, at, -q)
            grad[i:j][rows] = d * (s["grad_loss"][i:j].double()[rows][:, None] * case["inv_t"])
    return (loss, grad) if case["train"] else loss
