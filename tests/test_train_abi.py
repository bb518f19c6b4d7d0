"""The training calls of the C ABI on the host (no GPU needed): workspace
queries, and arguments rejected before any HIP call.  Pointers are fake: each
call is built so that a check rejects it."""
import ctypes

import pytest

import paper_2403_06988_amd as dv

lib = dv.lib
OK, INVALID, SHAPE, DTYPE, ALIAS, WORKSPACE, HIP = range(7)
P = 0x7F0000000000
GB = 1 << 30
BIG = 1 << 50


def head(x=P, ldx=64, w=P + GB, ldw=64, dt=1, N=8, D=64, V=1000, t=P + 2 * GB, al=None, S=0, st=None, loss=P + 5 * GB,
         lse=P + 6 * GB, ws=P + 7 * GB, nb=BIG):
    return lib.dv_head_loss(x, ldx, w, ldw, dt, N, D, V, t, al, S, st, loss, lse, ws, nb, None)


def head_back(x=P, ldx=64, w=P + GB, ldw=64, dt=1, N=8, D=64, V=1000, t=P + 2 * GB, al=None, S=0, st=None, lse=P + 5 * GB,
              g=P + 6 * GB, gx=P + 7 * GB, gw=P + 8 * GB, ws=P + 9 * GB, nb=BIG):
    return lib.dv_head_loss_backward(x, ldx, w, ldw, dt, N, D, V, t, al, S, st, lse, g, gx, gw, ws, nb, None)


HEAD = [
    (dict(w=None), INVALID), (dict(x=None), INVALID), (dict(t=None), INVALID),
    (dict(al=P + 3 * GB, S=2), INVALID), (dict(st=P + 3 * GB), INVALID), (dict(x=P + 1), INVALID),
    (dict(w=P + GB + 2, dt=0), INVALID),
    (dict(N=-1), SHAPE), (dict(N=(1 << 20) + 1), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1), SHAPE),
    (dict(D=0), SHAPE), (dict(D=65537, ldx=1 << 17, ldw=1 << 17), SHAPE), (dict(ldx=63), SHAPE), (dict(ldw=63), SHAPE),
    (dict(ldx=(1 << 40) + 1), SHAPE), (dict(al=P + 3 * GB, S=0, st=P + 4 * GB), SHAPE),
    (dict(al=P + 3 * GB, S=65536, st=P + 4 * GB), SHAPE),
    (dict(dt=2), DTYPE), (dict(dt=-1), DTYPE),
    (dict(ws=None), WORKSPACE), (dict(nb=64), WORKSPACE), (dict(ws=P + 7 * GB + 4), WORKSPACE),
]


@pytest.mark.parametrize("kw,status", HEAD + [
    (dict(loss=None), INVALID), (dict(lse=None), INVALID), (dict(loss=P + 6 * GB + 4), ALIAS), (dict(loss=P + 16), ALIAS),
    (dict(lse=P + GB + 64), ALIAS), (dict(lse=P + 2 * GB), ALIAS), (dict(ws=P + GB), ALIAS), (dict(ws=P + 5 * GB), ALIAS),
])
def test_head_loss_rejects_before_launch(kw, status):
    assert head(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_head_loss:")


@pytest.mark.parametrize("kw,status", HEAD + [
    (dict(lse=None), INVALID), (dict(g=None), INVALID), (dict(gx=None, gw=None), INVALID), (dict(gx=P + 7 * GB + 1), INVALID),
    (dict(gx=P), ALIAS), (dict(gw=P + GB), ALIAS), (dict(gw=P + 7 * GB + 128), ALIAS), (dict(gx=P + 6 * GB), ALIAS),
    (dict(ws=P + 8 * GB), ALIAS),
])
def test_head_loss_backward_rejects_before_launch(kw, status):
    if "nb" in kw:
        kw = dict(kw, ws=P + 9 * GB)
    elif kw.get("ws") == P + 7 * GB + 4:
        kw = dict(ws=P + 9 * GB + 4)
    assert head_back(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_head_loss_backward:")


def distill(z=P, ld=1000, dt=1, N=8, V=1000, ids=P + GB, top=P + 2 * GB, K=4, c=1.0, al=None, S=0, st=None, loss=P + 5 * GB,
            ws=P + 7 * GB, nb=BIG):
    return lib.dv_distill_loss(z, ld, dt, N, V, ids, top, K, c, al, S, st, loss, ws, nb, None)


def distill_back(z=P, ld=1000, dt=1, N=8, V=1000, ids=P + GB, top=P + 2 * GB, K=4, c=1.0, al=None, S=0, st=None,
                 g=P + 4 * GB, loss=P + 5 * GB, grad=P + 6 * GB, ldg=1000, ws=P + 7 * GB, nb=BIG):
    return lib.dv_distill_loss_backward(z, ld, dt, N, V, ids, top, K, c, al, S, st, g, loss, grad, ldg, ws, nb, None)


DISTILL = [
    (dict(z=None), INVALID), (dict(ids=None), INVALID), (dict(top=None), INVALID), (dict(z=P + 1), INVALID),
    (dict(al=P + 3 * GB, S=2), INVALID),
    (dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(K=0), SHAPE), (dict(K=1025), SHAPE), (dict(ld=999), SHAPE),
    (dict(c=0.0), SHAPE), (dict(c=-1.0), SHAPE), (dict(c=float("nan")), SHAPE), (dict(c=float("inf")), SHAPE),
    (dict(al=P + 3 * GB, S=-1, st=P + 3 * GB), SHAPE), (dict(dt=3), DTYPE),
    (dict(ws=None), WORKSPACE), (dict(nb=8), WORKSPACE), (dict(ws=P + 7 * GB + 128), WORKSPACE),
    (dict(loss=P + 64), ALIAS), (dict(loss=P + GB), ALIAS), (dict(ws=P + 2 * GB), ALIAS),
]


@pytest.mark.parametrize("kw,status", DISTILL + [(dict(loss=None), INVALID)])
def test_distill_loss_rejects_before_launch(kw, status):
    assert distill(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_distill_loss:")


@pytest.mark.parametrize("kw,status", DISTILL + [
    (dict(g=None), INVALID), (dict(grad=None), INVALID), (dict(grad=P + 6 * GB + 1), INVALID), (dict(ldg=999), SHAPE),
    (dict(grad=P + 2), ALIAS),                     # shifted over the logits
    (dict(grad=P, ldg=1008), ALIAS),               # over them with another stride
    (dict(grad=P + 5 * GB), ALIAS), (dict(grad=P + 4 * GB), ALIAS),
])
def test_distill_loss_backward_rejects_before_launch(kw, status):
    assert distill_back(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_distill_loss_backward:")


def embed(w=P, ld=64, dt=1, V=1000, D=64, ids=P + GB, N=8, scale=1.0, out=P + 2 * GB):
    return lib.dv_embed(w, ld, dt, V, D, ids, N, scale, out, None)


def embed_back(g=P, ld=64, dt=1, N=8, D=64, ids=P + GB, V=1000, scale=1.0, acc=0, gw=P + 2 * GB, ws=P + 3 * GB, nb=BIG):
    return lib.dv_embed_backward(g, ld, dt, N, D, ids, V, scale, acc, gw, ws, nb, None)


@pytest.mark.parametrize("kw,status", [
    (dict(w=None), INVALID), (dict(ids=None), INVALID), (dict(out=None), INVALID), (dict(out=P + 2 * GB + 1), INVALID),
    (dict(w=P + 2, dt=0), INVALID), (dict(V=0), SHAPE), (dict(D=0), SHAPE), (dict(N=-1), SHAPE), (dict(ld=63), SHAPE),
    (dict(scale=float("inf")), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(dt=9), DTYPE), (dict(out=P + 128), ALIAS),
    (dict(out=P + GB - 16), ALIAS),
])
def test_embed_rejects_before_launch(kw, status):
    assert embed(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_embed:")


@pytest.mark.parametrize("kw,status", [
    (dict(gw=None), INVALID), (dict(g=None), INVALID), (dict(ids=None), INVALID), (dict(gw=P + 2 * GB + 1), INVALID),
    (dict(V=0), SHAPE), (dict(D=70000, ld=70000), SHAPE), (dict(N=-1), SHAPE), (dict(ld=63), SHAPE),
    (dict(scale=float("-inf")), SHAPE), (dict(dt=9), DTYPE), (dict(gw=P), ALIAS), (dict(gw=P + GB), ALIAS),
    (dict(ws=None), WORKSPACE), (dict(nb=16), WORKSPACE), (dict(ws=P + 3 * GB + 1), WORKSPACE), (dict(ws=P + 2 * GB), ALIAS),
    (dict(ws=P + GB), ALIAS),
])
def test_embed_backward_rejects_before_launch(kw, status):
    assert embed_back(**kw) == status
    assert lib.dv_last_error().startswith(b"dv_embed_backward:")


def test_calls_without_rows_do_nothing():
    assert head(N=0, x=None, t=None, loss=None, lse=None, ws=None, nb=0) == OK
    assert head_back(N=0, x=None, t=None, lse=None, g=None, gx=None, gw=None, ws=None, nb=0) == OK
    assert distill(N=0, z=None, ids=None, top=None, loss=None, ws=None, nb=0) == OK
    assert distill_back(N=0, z=None, ids=None, top=None, g=None, loss=None, grad=None, ws=None, nb=0) == OK
    assert embed(N=0, ids=None, out=None) == OK
    assert embed_back(N=0, g=None, ids=None, acc=1) == OK
    assert lib.dv_last_error() == b""


def test_workspace_queries():
    q = lib.dv_head_loss_workspace_bytes
    assert q(-1, 64, 100, 1) == q(8, 0, 100, 1) == q(8, 64, 0, 1) == q(8, 64, 100, 2) == q((1 << 20) + 1, 64, 100, 1) == 0
    assert q(0, 64, 100, 1) > 0
    b = lib.dv_head_loss_backward_workspace_bytes
    assert b(8, 70000, 100, 1) == 0 and b(8, 64, 100, 0) > 0
    # the logits of 8,192 rows x 256,000 tokens would be 8.4 GB: the workspaces stay far below
    assert 0 < q(8192, 4096, 256000, 1) < 1 << 30
    assert 0 < b(8192, 4096, 256000, 1) < 3 << 30
    d = lib.dv_distill_loss_workspace_bytes
    assert d(8, 100, 0) == d(8, 100, 1025) == d(8, 0, 4) == d(-1, 100, 4) == 0
    sizes = [d(n, 128256, 64) for n in (0, 1, 2, 100, 255, 256, 1000, 1 << 20)]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))
    e = lib.dv_embed_backward_workspace_bytes
    assert e(8, 0, 100) == e(8, 64, 0) == 0 and e(0, 64, 100) > 0
    sizes = [e(n, 64, 100) for n in (0, 1, 100, 8192, 8193, 100000, 1 << 20)]
    assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))


def test_binding_refuses_host_tensors():
    import torch
    x, w, t = torch.zeros((2, 64)), torch.zeros((10, 64)), torch.zeros(2, dtype=torch.int32)
    for bad in (lambda: dv.head_loss(x, w, t), lambda: dv.embed(w, t), lambda: dv.embed_backward(x, t, 10),
                lambda: dv.distill_loss(x, torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3)))):
        with pytest.raises((TypeError, ValueError)):
            bad()


@pytest.mark.parametrize("call", [distill, distill_back])
def test_inverse_temperature_whose_exponent_is_not_finite(call):
    """The kernels scale by c log2(e) in fp32, infinite from 2.36e38 on."""
    assert call(c=2.4e38) == call(c=3.0e38) == call(c=3.4e38) == SHAPE
    assert b"inv_temperature" in lib.dv_last_error()
    assert call(c=2.3e38, ws=None) == WORKSPACE  # passes; the next check does not


def test_head_workspaces_hold_no_copy_that_is_not_made():
    """A call's own query: nothing for operands that are used where they lie.  Any
    operands' query: at most 2^27 elements of packed weights, and 2^19 a row."""
    MB = 1 << 20
    for dt, elt in ((1, 2), (0, 4)):
        for rows in (1, 8, 64):
            for D, V in ((4096, 128256), (4096, 256000), (1024, 1000000)):
                at = lambda q, x=P, ld_x=D, w=P + 64 * GB, ld_w=D: q(x, ld_x, w, ld_w, dt, rows, D, V)  # noqa: E731
                copies = ((1 << 27) + (rows << 19)) * elt + 64 * D * elt
                states, g = (V // 32 + 8) * rows * 8 + MB, min(V + 64, 1 << 18) * 64 * 4 + 64 * D * 16 * 4 + MB
                own, back = lib.dv_head_loss_workspace_bytes_for, lib.dv_head_loss_backward_workspace_bytes_for
                assert 0 < at(own) <= states and 0 < at(back) <= g
                assert at(own, w=P + 64 * GB + 16) == at(own)
                for kw in (dict(w=P + 64 * GB + 2 * elt), dict(ld_w=D + 1), dict(x=P + elt), dict(ld_x=D + 1), dict(ld_w=(1 << 20) + 64)):
                    assert at(own) < at(own, **kw) <= states + copies, kw
                    assert at(back) < at(back, **kw) <= g + copies, kw
                    assert at(own, **kw) <= lib.dv_head_loss_workspace_bytes(rows, D, V, dt) <= states + copies
                    assert at(back, **kw) <= lib.dv_head_loss_backward_workspace_bytes(rows, D, V, dt) <= g + copies
    # the states of 128-token tiles, not of 32-token ones
    assert own(P, 4096, P + 64 * GB, 4096, 1, 8192, 4096, 256000) < 8192 * (256000 // 128 + 2) * 8 + MB
    for bad in ((-1, 64, 100), (8, 0, 100), (8, 64, 0), (8, 70000, 100)):
        assert own(P, 1 << 17, P, 1 << 17, 1, *bad) == back(P, 1 << 17, P, 1 << 17, 1, *bad) == 0


def test_a_workspace_of_the_calls_own_size_is_taken():
    """Aligned operands pass with their own size; the same size with a stride that needs copies does not."""
    need = lib.dv_head_loss_workspace_bytes_for(P, 64, P + GB, 64, 1, 8, 64, 1000)
    assert head(nb=need - 1) == WORKSPACE and head(nb=need, loss=P + 16) == ALIAS
    assert head(nb=need, ldw=65) == head(nb=need, x=P + 2) == WORKSPACE
    need = lib.dv_head_loss_backward_workspace_bytes_for(P, 64, P + GB, 64, 1, 8, 64, 1000)
    assert head_back(nb=need - 1) == WORKSPACE and head_back(nb=need, gx=P) == ALIAS
    assert head_back(nb=need, ldw=65) == head_back(nb=need, x=P + 2) == WORKSPACE


def test_head_launches_stay_within_the_grid():
    """A launch has fewer than 2^32 threads, whatever the limits allow."""
    from tests.test_gpu_head_loss import plan_of
    import torch
    threads = {256: 512, 128: 256, 64: 256, 32: 128}

    def launch(i, j, side):
        other = 64 if side == 32 else side
        return -(-i // other) * -(-j // side) * threads[side]

    for dtype in (torch.bfloat16, torch.float32):
        for N in (1, 33, 8192, 100000, 300000, 1 << 20):
            for V in (1, 1000, 128256, 600000, 5000000, 1 << 24):
                for D in (1, 64, 4096, 65536):
                    for here in (False, True):
                        p = plan_of(N, D, V, dtype, here)
                        assert p.loss_tokens == V or p.loss_tokens % 256 == 0
                        k = (D + 63) // 64 * 64
                        for n in (launch(p.loss_tokens, N, p.loss_side), launch(p.piece_tokens, N, p.logits_side[0]),
                                  launch(k, N, p.grad_x_side), launch(k, p.piece_tokens, p.grad_weight_side[0])):
                            assert n < 1 << 32, (N, V, D, here)
