"""The training operators where arrays pass 2^31 elements, in HIP graphs, and on
streams of their own."""
import math

import pytest
import torch

from tests.train_common import check, distill_reference, head_reference

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def test_distill_past_two_to_the_31_elements(dv):
    N, V, K = 17000, 128256, 5
    assert N * V > 1 << 31
    print(f"distill N={N} V={V}", flush=True)
    g = gen(1)
    z = torch.empty((N, V), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    ids = torch.randint(0, V, (N, K), generator=g, device=DEV, dtype=torch.int32)
    top = torch.randn((N, K), generator=g, device=DEV)
    w = torch.randn(N, generator=g, device=DEV)
    loss, grad = dv.distill_loss_backward(z, ids, top, w)
    for n in (0, 8371, 16744, N - 1):  # below, around and past element 2^31
        ref = distill_reference(z[n:n + 1].cpu(), ids[n:n + 1].cpu(), top[n:n + 1].cpu(), 1.0,
                                torch.ones((1, V), dtype=torch.bool), w[n:n + 1].cpu())
        check(loss[n:n + 1], ref["loss"], ref["loss_tol"], f"loss {n}")
        check(grad[n:n + 1], ref["grad"], ref["grad_tol"], f"grad {n}")


def test_head_with_weights_past_two_to_the_31_elements(dv):
    N, D, V = 4, 4096, 530000
    assert V * D > 1 << 31
    print(f"head N={N} D={D} V={V}", flush=True)
    g = gen(2)
    w = torch.empty((V, D), dtype=torch.bfloat16, device=DEV).normal_(generator=g).mul_(1.0 / 64)
    x = torch.randn((N, D), generator=g, device=DEV).bfloat16()
    t = torch.tensor([0, 524287, 524289, V - 1], dtype=torch.int32, device=DEV)
    gl = torch.randn(N, generator=g, device=DEV)
    loss, lse = dv.head_loss(x, w, t)
    gx, gw = dv.head_loss_backward(x, w, t, lse, gl)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    # an fp32 sum of D terms, then of V
    tol = D * 2.0 ** -24 * (x.double().abs() @ w.double().abs().t()).max() + V * 2.0 ** -24
    assert (lse.double() - want).abs().max() < tol
    assert (loss.double() - (want - z[torch.arange(N), t.long()])).abs().max() < 2 * tol
    G = torch.softmax(z, 1)
    G[torch.arange(N), t.long()] -= 1
    G *= gl.double()[:, None]
    for v in (0, 1, 524287, 524288, 524289, V - 1):
        y = G[:, v] @ x.double()
        bound = (2.0 ** -8 + 2.0 ** -10) * (G[:, v].abs() @ x.double().abs()) + 2.0 ** -8 * y.abs()
        assert ((gw[v].double() - y).abs() <= bound).all(), v
    y = G @ w.double()
    bound = (2.0 ** -8 + 2.0 ** -10 + V * 2.0 ** -24) * (G.abs() @ w.double().abs()) + 2.0 ** -8 * y.abs()
    assert ((gx.double() - y).abs() <= bound).all()


def test_embedding_past_two_to_the_31_elements(dv):
    N, D, V = 300, 4096, 530000
    print(f"embed N={N} D={D} V={V}", flush=True)
    g = gen(3)
    w = torch.empty((V, D), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    ids = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    ids[:4] = torch.tensor([524287, 524288, 524289, V - 1], dtype=torch.int32)
    assert torch.equal(dv.embed(w, ids), w[ids.long()])
    go = torch.randn((N, D), generator=g, device=DEV).bfloat16()
    grad = dv.embed_backward(go, ids, V, grad_weight=w)  # over what was there
    want = torch.zeros((V, D), dtype=torch.float32, device=DEV).index_add_(0, ids.long(), go.float())
    assert (grad.float() - want).abs().max() <= 2.0 ** -8 * want.abs().max()
    present = torch.zeros(V, dtype=torch.bool, device=DEV)
    present[ids.long()] = True
    assert not grad[~present].any()


def test_row_strides_beyond_the_products_reach(dv):
    """Rows 2^20 elements apart and more are packed first."""
    N, D, V = 5, 64, 40
    g = gen(4)
    wide = torch.zeros((V, (1 << 20) + 64), dtype=torch.bfloat16, device=DEV)
    w = wide[:, :D]
    w.normal_(generator=g)
    x = torch.randn((N, D), generator=g, device=DEV).bfloat16()
    t = torch.arange(N, dtype=torch.int32, device=DEV)
    gl = torch.ones(N, device=DEV)
    loss, lse = dv.head_loss(x, w, t)
    near = dv.head_loss(x, w.contiguous(), t)
    assert torch.equal(loss, near[0]) and torch.equal(lse, near[1])
    ref = head_reference(x.cpu(), w.cpu(), t.cpu(), torch.ones((N, V), dtype=torch.bool), gl.cpu())
    gx, gw = dv.head_loss_backward(x, w, t, lse, gl)
    check(gx, ref["grad_x"], ref["grad_x_tol"], "grad_x")
    check(gw, ref["grad_weight"], ref["grad_weight_tol"], "grad_weight")


def _step(dv, N, D, V, K):
    """One training step with every buffer the caller's: (launches, outputs, inputs)."""
    g = gen(5)
    table = (torch.randn((V, D), generator=g, device=DEV) / math.sqrt(D)).bfloat16()
    ids = torch.randint(-1, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    t = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    z = torch.randn((N, V), generator=g, device=DEV).bfloat16()
    t_ids = torch.randint(0, V, (N, K), generator=g, device=DEV, dtype=torch.int32)
    top = torch.randn((N, K), generator=g, device=DEV)
    gl = torch.rand(N, generator=g, device=DEV)
    f32 = dict(dtype=torch.float32, device=DEV)
    o = dict(x=torch.empty((N, D), dtype=torch.bfloat16, device=DEV), loss=torch.empty(N, **f32), lse=torch.empty(N, **f32),
             gx=torch.empty((N, D), dtype=torch.bfloat16, device=DEV), gw=torch.empty_like(table),
             dl=torch.empty(N, **f32), gz=torch.empty_like(z))
    ws = torch.empty(max(dv.head_loss_workspace_bytes(N, D, V, torch.bfloat16),
                         dv.head_loss_backward_workspace_bytes(N, D, V, torch.bfloat16),
                         dv.distill_loss_workspace_bytes(N, V, K), dv.embed_backward_workspace_bytes(N, D, V)),
                     dtype=torch.uint8, device=DEV)

    def launches():
        dv.embed(table, ids, 2.0, out=o["x"])
        dv.head_loss(o["x"], table, t, loss=o["loss"], lse=o["lse"], workspace=ws)
        dv.head_loss_backward(o["x"], table, t, o["lse"], gl, grad_x=o["gx"], grad_weight=o["gw"], workspace=ws)
        dv.embed_backward(o["gx"], ids, V, 2.0, grad_weight=o["gw"], accumulate=True, workspace=ws)
        dv.distill_loss_backward(z, t_ids, top, gl, loss=o["dl"], grad=o["gz"], workspace=ws)

    return launches, o, (table, z, gl)


@pytest.mark.parametrize("N,D,V,K", [(100, 128, 3000, 8), (700, 256, 20000, 16), (20, 64, 140000, 30)])
def test_a_step_in_a_graph(dv, N, D, V, K):
    import bench
    print(f"graph N={N} D={D} V={V}", flush=True)
    launches, out, (table, z, gl) = _step(dv, N, D, V, K)
    launches()
    torch.cuda.synchronize()
    graph = bench.HipGraph(launches, DEV)
    try:
        for r in range(4):
            table.mul_(1.0 + 0.25 * r)  # new inputs in place, eager work between the replays
            z.add_(0.5)
            gl.mul_(-1.5)
            launches()
            torch.cuda.synchronize()
            want = {k: v.clone() for k, v in out.items()}
            for v in out.values():
                v.fill_(7)
            graph.replay()
            torch.cuda.synchronize()
            for k, v in out.items():
                assert torch.equal(v, want[k]), (r, k)
    finally:
        graph.close()


def test_a_step_on_another_stream(dv):
    launches, out, _ = _step(dv, 200, 128, 5000, 8)
    launches()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in out.items()}
    for v in out.values():
        v.fill_(3)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        launches()
    side.synchronize()
    for k, v in out.items():
        assert torch.equal(v, want[k]), k


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head_loss_in_several_launches(dv, dtype):
    """More tiles than one grid is given: the vocabulary in several launches, the weights in place."""
    N, D, V = 290001, 64, 70001
    from tests.test_gpu_head_loss import plan_of
    step = plan_of(N, D, V, dtype, True).loss_tokens
    assert step < V
    print(f"head N={N} D={D} V={V} {dtype} in launches of {step}", flush=True)
    g = gen(6)
    w = (torch.randn((V, D), generator=g, device=DEV) * 0.4).to(dtype)
    x = torch.randn((N, D), generator=g, device=DEV).to(dtype)
    t = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    pick = torch.arange(0, N, 1999, device=DEV)
    pick[-1] = N - 1
    t[pick[:4]] = torch.tensor([0, step - 1, step, V - 1], dtype=torch.int32, device=DEV)
    loss, lse = dv.head_loss(x, w, t)
    with torch.device(DEV):
        ref = head_reference(x[pick], w, t[pick], torch.ones((len(pick), V), dtype=torch.bool))
    for got, name in ((loss, "loss"), (lse, "lse")):
        check(got[pick], ref[name].cpu(), ref[name + "_tol"].cpu(), name)
