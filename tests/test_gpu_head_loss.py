"""dv_head_loss and its backward pass against their 64-bit forms, element by
element within derived bounds; gradients also against differences of the
loss; edges of masks, targets, strides and sizes; refusals."""
import ctypes
import math
import os

import numpy as np
import pytest
import torch

from tests.train_common import check, head_reference, masks, pack_mask, row_mask

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def on_device(t, pad):
    """t on the device with rows `pad` elements further apart, the first off a 16-byte boundary when pad is odd."""
    if pad == 0:
        return t.to(DEV)
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=DEV)
    view = wide[:, pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t)
    return view


def make(seed, N, D, V, dtype, S, shares=(0.0, 0.02, 0.5, 1.0), std=3.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.normal(size=(N, D))).to(dtype)
    w = torch.from_numpy(rng.normal(size=(V, D)) * std / math.sqrt(D)).to(dtype)
    may = masks(rng, S, V, shares) if S else None
    states = torch.from_numpy(rng.integers(-1, S + 1, N).astype(np.int32)) if S else None
    mask = row_mask(may, states, N, V)
    targets = torch.zeros(N, dtype=torch.int32)
    for n in range(N):
        allowed = torch.nonzero(mask[n])[:, 0]
        if allowed.numel() and n % 7:
            targets[n] = int(allowed[rng.integers(allowed.numel())])
        else:  # padding, past the end, or any token
            targets[n] = [-1, V, -2147483648, int(rng.integers(V))][rng.integers(4)]
    g = torch.from_numpy(rng.normal(size=N)).float()
    return x, w, targets, may, states, mask, g


def run(dv, x, w, targets, may, states, g, pad=0):
    kw = {}
    if may is not None:
        kw = dict(allow=pack_mask(may).to(DEV), states=states.to(DEV))
    xd, wd, td = on_device(x, pad), on_device(w, pad), targets.to(DEV)
    loss, lse = dv.head_loss(xd, wd, td, **kw)
    gx, gw = dv.head_loss_backward(xd, wd, td, lse, g.to(DEV), **kw)
    torch.cuda.synchronize()
    return loss, lse, gx, gw


# rows, hidden, tokens: one of each, below and above the tiles' sides and their k, odd ones
SIZES = [(1, 1, 1), (1, 64, 32), (2, 8, 33), (3, 65, 100), (17, 100, 257), (64, 64, 256), (65, 128, 255), (33, 192, 1000),
         (130, 63, 513), (200, 256, 300), (300, 72, 2049)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("N,D,V", SIZES)
def test_matches_the_64_bit_form(dv, N, D, V, dtype, masked):
    print(f"head N={N} D={D} V={V} {dtype} masked={masked}", flush=True)
    x, w, t, may, states, mask, g = make(N * 7 + D + V, N, D, V, dtype, 5 if masked else 0)
    ref = head_reference(x, w, t, mask, g)
    for pad in (0, 3):
        loss, lse, gx, gw = run(dv, x, w, t, may, states, g, pad)
        check(lse, ref["lse"], ref["lse_tol"], "lse")
        check(loss, ref["loss"], ref["loss_tol"], "loss")
        check(gx, ref["grad_x"], ref["grad_x_tol"], "grad_x")
        check(gw, ref["grad_weight"], ref["grad_weight_tol"], "grad_weight")
        assert gx.dtype == dtype and gw.dtype == dtype


@pytest.mark.parametrize("N,D,V,dtype", [
    (700, 640, 5000, torch.bfloat16),     # 128-sided tiles, split k
    (2100, 512, 6200, torch.bfloat16),    # 256-sided tiles
    (1100, 256, 5003, torch.float32),
])
def test_larger_tiles(dv, N, D, V, dtype):
    print(f"head large N={N} D={D} V={V} {dtype}", flush=True)
    x, w, t, may, states, mask, g = make(3, N, D, V, dtype, 6)
    ref = head_reference(x, w, t, mask, g)
    loss, lse, gx, gw = run(dv, x, w, t, may, states, g)
    check(lse, ref["lse"], ref["lse_tol"], "lse")
    check(loss, ref["loss"], ref["loss_tol"], "loss")
    check(gx, ref["grad_x"], ref["grad_x_tol"], "grad_x")
    check(gw, ref["grad_weight"], ref["grad_weight_tol"], "grad_weight")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_several_pieces_of_the_vocabulary(dv, dtype):
    """More rows than a piece of the vocabulary covers in one go."""
    N, D, V = 20000, 64, 9000
    print(f"head pieces N={N} D={D} V={V} {dtype}", flush=True)
    assert N * V > 1 << 27
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((N, D), generator=g, device=DEV).to(dtype)
    w = (torch.randn((V, D), generator=g, device=DEV) * 0.3).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    gl = torch.randn(N, generator=g, device=DEV)
    loss, lse = dv.head_loss(x, w, t)
    gx, gw = dv.head_loss_backward(x, w, t, lse, gl)
    pick = torch.arange(0, N, 997)
    ref = head_reference(x[pick].cpu(), w.cpu(), t[pick].cpu(), torch.ones((len(pick), V), dtype=torch.bool), gl[pick].cpu())
    check(loss[pick], ref["loss"], ref["loss_tol"], "loss")
    check(lse[pick], ref["lse"], ref["lse_tol"], "lse")
    check(gx[pick], ref["grad_x"], ref["grad_x_tol"], "grad_x")
    # the weight's gradient takes every row: its sums against those over float64 on the device, whole
    z = x.double() @ w.double().t()
    G = torch.softmax(z, 1)
    G[torch.arange(N, device=DEV), t.long()] -= 1
    G *= gl.double()[:, None]
    want = G.t().contiguous() @ x.double()
    mags = G.abs().t().contiguous() @ x.double().abs()
    # the terms' error (2^-8 of bf16 G; fp32: logits within 2^-14 of e) and N terms' sum
    term = 2.0 ** -8 + 2.0 ** -12 if dtype == torch.bfloat16 else 2.0 ** -13
    out = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    tol = (term + 6 * N * 2.0 ** -24) * mags + out * want.abs()
    check(gw, want.cpu(), tol.cpu(), "grad_weight")


def test_gradient_against_differences(dv):
    N, D, V = 6, 24, 70
    x, w, t, may, states, mask, g = make(11, N, D, V, torch.float32, 4, shares=(0.6, 1.0))
    t = t.clamp(0, V - 1)
    kw = dict(allow=pack_mask(may).to(DEV), states=states.to(DEV))
    g = g.to(DEV)

    def total(x, w):
        loss, lse = dv.head_loss(x.to(DEV), w.to(DEV), t.to(DEV), **kw)
        return float((loss.double() * g.double()).sum()), lse

    _, lse = total(x, w)
    gx, gw = dv.head_loss_backward(x.to(DEV), w.to(DEV), t.to(DEV), lse, g, **kw)
    rng = np.random.default_rng(2)
    for _ in range(6):
        dx = torch.from_numpy(rng.normal(size=x.shape)).float()
        dw = torch.from_numpy(rng.normal(size=w.shape)).float()
        h = 2.0 ** -7
        diff = (total(x + h * dx, w + h * dw)[0] - total(x - h * dx, w - h * dw)[0]) / (2 * h)
        along = float((gx.cpu().double() * dx.double()).sum() + (gw.cpu().double() * dw.double()).sum())
        # third derivatives of the loss along (dx, dw) times h^2 / 6, and the losses' rounding over 2 h
        assert abs(diff - along) < 0.02 * (1 + abs(along)), (diff, along)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rows_that_take_no_part(dv, dtype):
    """Empty masks, dead states, targets that are padding or not allowed: loss
    0, no gradient, and no trace of them in the others' gradients."""
    N, D, V = 40, 64, 300
    x, w, t, may, states, mask, g = make(21, N, D, V, dtype, 3, shares=(0.0, 1.0, 0.3))
    states[:] = 1
    states[3], states[4], states[5] = 0, -1, 77
    t[:] = 5
    t[6], t[7] = -1, V
    states[8] = 2
    t[8] = int(torch.nonzero(~may[2])[0, 0])
    out = [3, 4, 5, 6, 7, 8]
    loss, lse, gx, gw = run(dv, x, w, t, may, states, g)
    assert torch.equal(loss[out].cpu(), torch.zeros(len(out)))
    assert torch.equal(gx[out].float().cpu(), torch.zeros((len(out), D)))
    assert bool((lse[[3, 4, 5]] == -math.inf).all()) and bool(torch.isfinite(lse[[6, 7, 8]]).all())
    keep = [n for n in range(N) if n not in out]
    ref = head_reference(x, w, t, row_mask(may, states, N, V), g)
    check(gw, ref["grad_weight"], ref["grad_weight_tol"], "grad_weight")
    check(gx[keep], ref["grad_x"][keep], ref["grad_x_tol"][keep], "grad_x")
    # all of them: zeros everywhere
    loss, lse, gx, gw = run(dv, x, w, torch.full_like(t, -1), may, states, g)
    assert not loss.any() and not gx.any() and not gw.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_is_masked_has_no_effect(dv, dtype):
    """Weight rows that make masked logits huge change nothing; logits beyond
    exp's range on allowed tokens stay exact."""
    N, D, V = 9, 64, 200
    x, w, t, may, states, mask, g = make(31, N, D, V, dtype, 1, shares=(0.5,))
    states[:] = 0
    allowed = torch.nonzero(may[0])[:, 0]
    t[:] = int(allowed[0])
    x[0] *= 60  # logits of several hundred
    first = run(dv, x, w, t, may, states, g)
    w2 = w.clone()
    w2[~may[0]] *= 1e30
    second = run(dv, x, w2, t, may, states, g)
    assert torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    ref = head_reference(x, w, t, row_mask(may, states, N, V), g)
    check(first[0], ref["loss"], ref["loss_tol"], "loss")
    assert torch.equal(first[3][~may[0]], torch.zeros_like(first[3][~may[0]]))
    assert torch.equal(first[3][may[0]], second[3][may[0]])


def test_nan_is_seen(dv):
    N, D, V = 5, 64, 100
    x, w, t, may, states, mask, g = make(41, N, D, V, torch.float32, 0)
    t[:] = 1
    x[2] = float("nan")
    loss, lse, gx, gw = run(dv, x, w, t, None, None, g)
    assert bool(torch.isnan(loss[2])) and bool(torch.isnan(lse[2]))
    assert bool(torch.isfinite(loss[[0, 1, 3, 4]]).all())


def test_one_gradient_alone_and_no_rows(dv):
    N, D, V = 50, 96, 500
    x, w, t, may, states, mask, g = make(51, N, D, V, torch.bfloat16, 0)
    loss, lse, gx, gw = run(dv, x, w, t, None, None, g)
    args = (x.to(DEV), w.to(DEV), t.to(DEV), lse, g.to(DEV))
    ax, none = dv.head_loss_backward(*args, want_weight=False)
    assert none is None and torch.equal(ax, gx)
    none, aw = dv.head_loss_backward(*args, want_x=False)
    assert none is None and torch.equal(aw, gw)
    e = torch.empty((0, D), dtype=torch.bfloat16, device=DEV)
    none_t = torch.empty(0, dtype=torch.int32, device=DEV)
    none_f = torch.empty(0, device=DEV)
    loss, lse = dv.head_loss(e, w.to(DEV), none_t)
    assert loss.numel() == 0
    gw.fill_(7)
    gx, gw = dv.head_loss_backward(e, w.to(DEV), none_t, none_f, none_f, grad_weight=gw)
    assert gx.shape == (0, D) and not gw.any()


def test_same_bits_each_time_and_on_another_stream(dv):
    x, w, t, may, states, mask, g = make(61, 300, 256, 3000, torch.bfloat16, 4)
    first = run(dv, x, w, t, may, states, g)
    side = torch.cuda.Stream()
    kw = dict(allow=pack_mask(may).to(DEV), states=states.to(DEV))
    xd, wd, td, gd = x.to(DEV), w.to(DEV), t.to(DEV), g.to(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        loss, lse = dv.head_loss(xd, wd, td, **kw)
        gx, gw = dv.head_loss_backward(xd, wd, td, lse, gd, **kw)
    torch.cuda.synchronize()
    for a, b in zip(first, (loss, lse, gx, gw)):
        assert torch.equal(a, b)


def test_refusals(dv):
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    w = torch.zeros((100, 64), dtype=torch.bfloat16, device=DEV)
    t = torch.zeros(4, dtype=torch.int32, device=DEV)
    al = torch.zeros((2, 4), dtype=torch.int32, device=DEV)
    for bad in (lambda: dv.head_loss(x.half(), w.half(), t), lambda: dv.head_loss(x, w.float(), t),
                lambda: dv.head_loss(x, w, t.long()), lambda: dv.head_loss(x, w, t[:3]),
                lambda: dv.head_loss(x[:, :32], w, t), lambda: dv.head_loss(x.t(), w, t),
                lambda: dv.head_loss(x, w, t, allow=al), lambda: dv.head_loss(x, w, t, allow=al[:, :3], states=t),
                lambda: dv.head_loss(x, w, t, workspace=torch.zeros(16, dtype=torch.uint8, device=DEV)),
                lambda: dv.head_loss_backward(x, w, t, torch.zeros(3, device=DEV), torch.zeros(4, device=DEV)),
                lambda: dv.head_loss_backward(x, w, t, torch.zeros(4, device=DEV), torch.zeros(4, device=DEV),
                                              grad_x=torch.zeros((4, 32), dtype=torch.bfloat16, device=DEV))):
        with pytest.raises((TypeError, ValueError)):
            bad()
    with pytest.raises(dv.DvError):  # an output over an input
        dv.head_loss_backward(x, w, t, torch.zeros(4, device=DEV), torch.zeros(4, device=DEV), grad_x=x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_few_rows_beside_a_large_table_take_little_memory(dv, dtype):
    """Operands in place: no room for a copy of them; in a wider buffer: a piece's."""
    N, D, V = 2, 1024, 200000
    wide = torch.empty((V, D + 1), dtype=dtype, device=DEV).normal_()
    table = wide[:, :D].contiguous()
    x = torch.randn((N, D), device=DEV).to(dtype)
    t = torch.tensor([0, V - 1], dtype=torch.int32, device=DEV)
    gl = torch.ones(N, device=DEV)
    gx, gw = torch.empty_like(x), torch.empty_like(table)

    def most(w):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        loss, lse = dv.head_loss(x, w, t)
        dv.head_loss_backward(x, w, t, lse, gl, grad_x=gx, grad_weight=gw)
        torch.cuda.synchronize()
        return torch.cuda.max_memory_allocated() - before, loss, lse, gx.clone(), gw.clone()

    aligned, packed = most(table), most(wide[:, :D])
    g = 64 * (V + 64) * table.element_size()  # a piece of G for 64 rows
    assert aligned[0] < g + (8 << 20)
    assert packed[0] < g + (8 << 20) + ((1 << 27) + (N << 19)) * table.element_size()
    assert dv.head_loss_workspace_bytes_for(x, table) < dv.head_loss_workspace_bytes_for(x, wide[:, :D])
    assert dv.head_loss_workspace_bytes_for(x, wide[:, :D]) <= dv.head_loss_workspace_bytes(N, D, V, dtype)
    assert dv.head_loss_backward_workspace_bytes_for(x, table) < dv.head_loss_backward_workspace_bytes(N, D, V, dtype)
    for a, b in zip(aligned[1:3], packed[1:3]):
        assert torch.equal(a, b)  # the same tiles' sums


# ------------------------------------------------ every tile, split and piece

class Plan(ctypes.Structure):
    """struct dvprobe_head_plan"""
    _fields_ = [(n, ctypes.c_int32) for n in ("loss_tokens", "loss_side", "pieces", "piece_tokens", "last_piece_tokens")] + [
        ("logits_side", ctypes.c_int32 * 2), ("grad_x_side", ctypes.c_int32), ("grad_x_splits", ctypes.c_int32),
        ("grad_weight_side", ctypes.c_int32 * 2), ("grad_weight_splits", ctypes.c_int32 * 2)]


def plan_of(N, D, V, dtype, in_place):
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2403_06988_amd", "libdv_probes.so"))
    p = Plan()
    assert lib.dvprobe_head_plan(N, D, V, 1 if dtype == torch.bfloat16 else 0, in_place, in_place, ctypes.byref(p)) == 0
    return p


def make_on_device(seed, N, D, V, dtype, few, pad):
    """Masks from nothing over `few` tokens in a thousand to everything, dead rows, padding.
    Most rows' losses have no weight, and many rows few allowed tokens: a misplaced
    row or token then is no small part of the sums that it misses or spoils."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = on_device(torch.randn((N, D), generator=g, device=DEV).to(dtype), pad)
    w = on_device((torch.randn((V, D), generator=g, device=DEV) * (3.0 / math.sqrt(D))).to(dtype), pad)
    shares = torch.tensor([0.0, few / 1000, few / 1000, 0.3, 1.0], device=DEV)
    may = torch.rand((5, V), generator=g, device=DEV) < shares[:, None]
    states = torch.randint(-1, 6, (N,), generator=g, device=DEV, dtype=torch.int32)
    states[-1] = 1
    alive = (states >= 0) & (states < 5)
    mask = may[states.clamp(0, 4).long()] & alive[:, None]
    score = torch.rand((N, V), generator=g, device=DEV).masked_fill_(~mask, -1.0)
    t = score.argmax(1).int()  # an allowed token of each row that has one
    del score
    at = torch.arange(N, device=DEV)
    t[at % 11 == 3] = torch.tensor([-1, V, -2147483648], dtype=torch.int32, device=DEV)[at[at % 11 == 3] % 3]
    gl = torch.randn(N, generator=g, device=DEV)
    gl[(at % 29 != 0) & (at < N - 3)] = 0
    return x, w, t, may, states, mask, gl


def check_on_device(dv, x, w, t, may, states, mask, gl):
    kw = dict(allow=pack_mask(may.cpu()).to(DEV), states=states)
    loss, lse = dv.head_loss(x, w, t, **kw)
    gx, gw = dv.head_loss_backward(x, w, t, lse, gl, **kw)
    with torch.device(DEV):
        ref = {k: v.cpu() for k, v in head_reference(x, w, t, mask, gl).items()}
    check(lse, ref["lse"], ref["lse_tol"], "lse")
    check(loss, ref["loss"], ref["loss_tol"], "loss")
    check(gx, ref["grad_x"], ref["grad_x_tol"], "grad_x")
    check(gw, ref["grad_weight"], ref["grad_weight_tol"], "grad_weight")


BF, F = torch.bfloat16, torch.float32
# rows, hidden, tokens, row stride beyond hidden; then what the case is there for: the side of
# grad_x's tiles, whether its sum is split, several pieces; the same of grad_weight's
PLANS = [
    (BF, 2100, 2001, 501, 0, (128, False, False), (64, True)), (BF, 4000, 99, 17003, 0, (128, True, False), (128, True)),
    (BF, 20000, 999, 9001, 0, (128, False, True), (256, True)), (BF, 2100, 2001, 9001, 0, (256, True, False), (128, False)),
    (BF, 2100, 2048, 9001, 0, (256, True, False), (128, False)), (BF, 9000, 1499, 2003, 0, (256, False, False), (256, True)),
    (BF, 9000, 501, 17001, 0, (256, True, True), (256, True)), (BF, 9000, 1499, 17001, 0, (256, False, True), (256, False)),
    (BF, 9000, 1536, 17001, 0, (256, False, True), (256, False)), (BF, 300, 250, 50257, 3, (64, True, False), (256, False)),
    (BF, 6000, 99, 9001, 0, (128, True, False), (128, True)), (BF, 40, 99, 33001, 0, (64, True, False), (128, False)),
    (F, 2100, 2001, 501, 0, (128, False, False), (64, True)), (F, 9000, 99, 2003, 0, (128, True, False), (64, True)),
    (F, 2100, 4001, 501, 0, (256, False, False), (128, True)), (F, 700, 4001, 2003, 0, (256, True, False), (128, False)),
    (F, 700, 4096, 2003, 0, (256, True, False), (128, False)), (F, 9000, 249, 17001, 0, (256, True, True), (256, True)),
    (F, 9000, 1499, 17001, 0, (256, False, True), (256, True)), (F, 9000, 1536, 17001, 0, (256, False, True), (256, True)),
    (F, 40, 250, 33001, 3, (64, True, False), (256, False)), (F, 1100, 250, 17001, 0, (128, True, False), (256, True)),
    (F, 1500, 99, 9001, 0, (64, True, False), (128, True)), (F, 40, 99, 33001, 0, (64, True, False), (128, False)),
]


@pytest.mark.parametrize("dtype,N,D,V,pad,grad_x,grad_weight", PLANS)
def test_every_tile_and_split_of_the_gradients(dv, dtype, N, D, V, pad, grad_x, grad_weight):
    print(f"head plan N={N} D={D} V={V} {dtype}", flush=True)
    p = plan_of(N, D, V, dtype, D % 64 == 0 and pad == 0)
    assert (p.grad_x_side, p.grad_x_splits > 1, p.pieces > 1) == grad_x
    assert (p.grad_weight_side[0], p.grad_weight_splits[0] > 1) == grad_weight
    check_on_device(dv, *make_on_device(N + D, N, D, V, dtype, 3, pad))


@pytest.mark.parametrize("dtype,N,D,V,pad", [
    (BF, 9, 65, 262501, 0), (F, 9, 65, 262501, 0),        # pieces of 2^18 tokens at most
    (BF, 9, 4100, 70001, 0), (F, 9, 4096, 70001, 1),      # of 2^27 packed elements
    (BF, 4200, 33, 33003, 0), (F, 4200, 64, 33003, 3),    # of 2^27 logits
])
def test_several_packed_pieces(dv, dtype, N, D, V, pad):
    """Weights that are copied a piece at a time, in the loss too: each piece's
    place among masks, targets and partial results."""
    print(f"head packed pieces N={N} D={D} V={V} {dtype}", flush=True)
    p = plan_of(N, D, V, dtype, False)
    assert p.pieces > 1 and p.loss_tokens == p.piece_tokens and p.last_piece_tokens < p.piece_tokens
    x, w, t, may, states, mask, gl = make_on_device(D, N, D, V, dtype, 3, pad)
    # targets on both sides of each piece's end, and at the vocabulary's ends
    ends = [0, V - 1] + [v for i in range(1, p.pieces) for v in (i * p.piece_tokens - 1, i * p.piece_tokens)]
    assert len(ends) < N
    may[1:, ends] = True
    states[:len(ends)] = torch.arange(len(ends), dtype=torch.int32, device=DEV) % 4 + 1
    t[:len(ends)] = torch.tensor(ends, dtype=torch.int32, device=DEV)
    states[-2], states[-1] = 0, -1
    gl[:len(ends)] = 1.0
    mask = may[states.clamp(0, 4).long()] & ((states >= 0) & (states < 5))[:, None]
    check_on_device(dv, x, w, t, may, states, mask, gl)


def test_plans_of_the_measured_range():
    """The query itself: sides and pieces as the kernels have them, refusals."""
    for dtype in (BF, F):
        for N, D, V in ((1, 1024, 32000), (8192, 4096, 128256), (1999, 1000, 32003), (1 << 20, 64, 5000)):
            p = plan_of(N, D, V, dtype, False)
            assert p.loss_side in (32, 64, 128, 256) and p.grad_x_side in (32, 64, 128, 256)
            assert set(p.grad_weight_side) | set(p.logits_side) <= {32, 64, 128, 256}
            assert (p.pieces - 1) * p.piece_tokens + p.last_piece_tokens == V and 0 < p.last_piece_tokens <= p.piece_tokens
            assert plan_of(N, D, V, dtype, True).loss_tokens == V
    lib = ctypes.CDLL(os.path.join(ROOT, "paper_2403_06988_amd", "libdv_probes.so"))
    assert lib.dvprobe_head_plan(0, 8, 8, 1, 1, 1, ctypes.byref(Plan())) == 1
    assert lib.dvprobe_head_plan(8, 8, 8, 2, 1, 1, ctypes.byref(Plan())) == 1
    assert lib.dvprobe_head_plan(8, 8, 8, 1, 1, 1, None) == 1


@pytest.mark.parametrize("value", [math.inf, -math.inf, 3.4e38])
@pytest.mark.parametrize("N", [40, 1200])
def test_fp32_elements_beyond_the_range_stay_in_their_row(dv, value, N):
    """Infinite or nearly so: NaN for the row (or the rows that allow the token), and not a bit elsewhere."""
    D, V = 100, 700
    x, w, t, may, states, mask, g = make(71, N, D, V, F, 3, shares=(0.5, 1.0, 0.3))
    kw = dict(allow=pack_mask(may).to(DEV), states=states.to(DEV))
    t = t.to(DEV)
    clean = dv.head_loss(x.to(DEV), w.to(DEV), t, **kw)
    bad = x.clone()
    at = int(torch.nonzero((clean[0].cpu() != 0))[3, 0])
    bad[at, 17] = value
    got = dv.head_loss(bad.to(DEV), w.to(DEV), t, **kw)
    rest = torch.arange(N, device=DEV) != at
    for a, b in zip(got, clean):
        assert bool(torch.isnan(a[at])) and torch.equal(a[rest], b[rest])
    v = int(torch.nonzero(~may[0] & ~may[2])[0, 0])
    bad = w.clone()
    bad[v, 99] = value
    got = dv.head_loss(x.to(DEV), bad.to(DEV), t, **kw)
    sees = mask[:, v].to(DEV)
    assert sees.any() and not sees.all()
    assert bool(torch.isnan(got[1][sees]).all())
    for a, b in zip(got, clean):
        assert torch.equal(a[~sees], b[~sees])


@pytest.mark.parametrize("N,D,V,S,std", [
    (1, 64, 300, 0, 3.0), (5, 100, 700, 4, 3.0), (31, 128, 1000, 3, 1.0), (33, 256, 513, 0, 6.0), (70, 72, 2049, 4, 3.0),
    (300, 640, 3001, 4, 3.0), (1100, 512, 6200, 3, 0.5), (2100, 1024, 5000, 0, 3.0),
])
def test_bf16_gradients_are_rounded_once(dv, N, D, V, S, std):
    """Nothing on the way to the gradients is held in fewer bits than the sums:
    what is left is the stored results' own rounding.  The bounds are those of fp32
    inputs (their products' terms exceed what 16 bits of G leave out) and that rounding."""
    print(f"head bf16 gradients N={N} D={D} V={V} std={std}", flush=True)
    x, w, t, may, states, mask, g = make(N + D, N, D, V, BF, S, shares=(0.5, 0.01, 1.0, 0.1), std=std)
    loss, lse, gx, gw = run(dv, x, w, t, may, states, g)
    ref = head_reference(x.float(), w.float(), t, mask, g)
    for got, name in ((gx, "grad_x"), (gw, "grad_weight")):
        want = ref[name]
        check(got, want, ref[name + "_tol"] + 2.0 ** -8 * want.abs(), name)
        if want.any():
            off = lambda y: float((y.cpu().double() - want).norm() / want.norm())  # noqa: E731
            assert off(got) <= 1.02 * off(want.to(BF)) + 2.0 ** -16, name
