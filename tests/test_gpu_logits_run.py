"""The operators from the last layer to the logits together, as they are used:
a decode step, a captured one, a training step; on named streams; two at once."""
import numpy as np
import pytest
import torch

from tests.logits_common import norm_backward_reference, product_reference, quantize, values
from tests.train_common import check, masks, pack_mask

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def serving(rng, B=9, D=520, V=5003, H=60, S=12):
    t = lambda a, d=BF: torch.from_numpy(np.asarray(a)).to(d).to(DEV)  # noqa: E731
    may = masks(rng, S, V, [0.3, 0.9, 0.02, 0.0])
    ns = torch.where(may, torch.from_numpy(rng.integers(0, S, (S, V))), torch.tensor(-1)).to(torch.int32).to(DEV)
    return dict(x=t(rng.normal(size=(B, D))), residual=t(rng.normal(size=(B, D))), gain=t(rng.normal(size=D)),
                head=t(rng.normal(size=(V, D))), history=t(rng.integers(0, V, (B, H)), torch.int32),
                lengths=t(rng.integers(0, H + 1, B), torch.int32), repetition=t(1 + rng.random(B), F32),
                presence=t(rng.random(B), F32), frequency=t(rng.random(B), F32),
                bias_ids=t(rng.integers(-1, V, (B, 5)), torch.int32), bias=t(rng.normal(size=(B, 5)) * 9, F32),
                allow=pack_mask(may).to(DEV), next_state=ns, states=t(rng.integers(-1, S, B), torch.int32))


def decode(dv, s, head, head_scales, masked, **kw):
    """One step: (x + residual, adjusted logits, tokens, new states)."""
    q, scales, total = dv.rms_norm_f8(s["x"], s["gain"], 1e-5, residual=s["residual"], **kw)
    z = dv.product_f8(q, scales, head, head_scales, **kw)
    mask = dict(allow=s["allow"], states=s["states"]) if masked else {}
    dv.adjust_logits(z, s["history"], s["lengths"], repetition=s["repetition"], presence=s["presence"],
                     frequency=s["frequency"], bias_ids=s["bias_ids"], bias=s["bias"], out=z, **mask, **kw)
    token, new = dv.masked_step(s["next_state"], s["allow"], s["states"], z, **kw)
    return total, z, token, new


def test_a_decode_step(dv):
    """The logits within their bound of the 64-bit product of what the norm gave; the masked
    step chooses the same from masked logits and from logits with penalties alone."""
    s = serving(np.random.default_rng(1))
    head, hs, _, _ = dv.quantize_f8(s["head"], tile=128)
    q, scales, total = dv.rms_norm_f8(s["x"], s["gain"], 1e-5, residual=s["residual"])
    want, tol = product_reference(q.cpu(), scales.cpu(), head.cpu(), hs.cpu(), 128, BF)
    check(dv.product_f8(q, scales, head, hs), want, tol, "logits")
    t1, z1, tok1, new1 = decode(dv, s, head, hs, False)
    t2, z2, tok2, new2 = decode(dv, s, head, hs, True)
    assert torch.equal(t1, total) and torch.equal(t2, total)
    assert torch.equal(tok1, tok2) and torch.equal(new1, new2)
    live = z2 != -float("inf")
    assert torch.equal(z1[live], z2[live])
    for b in range(z2.shape[0]):
        assert (int(tok2[b]) == -1) == (not bool(live[b].any()))
        if int(tok2[b]) >= 0:
            assert int(tok2[b]) == int(torch.nonzero(z2[b] == z2[b].max())[0])


def test_a_captured_decode_step(dv):
    """Replays with eager work and other inputs between them, each equal to the eager call."""
    rng = np.random.default_rng(2)
    s = serving(rng)
    head, hs, _, _ = dv.quantize_f8(s["head"], tile=128)
    ws = dv.step_workspace(s["x"].shape[0], s["head"].shape[0], DEV)
    decode(dv, s, head, hs, True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, scales, total = dv.rms_norm_f8(s["x"], s["gain"], 1e-5, residual=s["residual"])
        z = dv.product_f8(q, scales, head, hs)
        dv.adjust_logits(z, s["history"], s["lengths"], repetition=s["repetition"], bias_ids=s["bias_ids"], bias=s["bias"],
                         allow=s["allow"], states=s["states"], out=z)
        token, new = dv.masked_step(s["next_state"], s["allow"], s["states"], z, workspace=ws)
    for k in range(4):
        s["x"].copy_(torch.from_numpy(rng.normal(size=tuple(s["x"].shape))))
        s["lengths"].copy_(torch.from_numpy(rng.integers(0, 61, s["lengths"].shape[0])))
        q2, sc2, total2 = dv.rms_norm_f8(s["x"], s["gain"], 1e-5, residual=s["residual"])
        z2 = dv.product_f8(q2, sc2, head, hs)
        z2 = dv.adjust_logits(z2, s["history"], s["lengths"], repetition=s["repetition"], bias_ids=s["bias_ids"],
                              bias=s["bias"], allow=s["allow"], states=s["states"])
        tok2, new2 = dv.masked_step(s["next_state"], s["allow"], s["states"], z2)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in ((total, total2), (q.view(torch.uint8), q2.view(torch.uint8)), (scales, sc2), (z, z2), (token, tok2),
                     (new, new2)):
            assert torch.equal(a, b), k


def test_captured_gradients(dv):
    rng = np.random.default_rng(3)
    t = lambda *shape: torch.from_numpy(rng.normal(size=shape)).to(BF).to(DEV)  # noqa: E731
    N, D, V = 200, 264, 700
    x, w, head, gz = t(N, D), t(D), t(V, D), t(N, V)

    def step():
        y, _, r = dv.rms_norm(x, w, 1e-5, want_rstd=True)
        q, s, tq, ts = dv.quantize_f8(y, want_columns=True)
        hq, hs, htq, hts = dv.quantize_f8(head, tile=128, want_columns=True)
        z = dv.product_f8(q, s, hq, hs)
        gq, gs, gtq, gts = dv.quantize_f8(gz, want_columns=True)
        gy = dv.product_f8(gq, gs, htq, hts)
        gw = dv.product_f8(gtq, gts, tq, ts, tile=1)
        return (z, gw, *dv.rms_norm_backward(gy, x, w, r))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(t(N, D))
        gz.copy_(t(N, V))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), k


@pytest.mark.parametrize("as_handle", [False, True])
def test_arrays_come_from_the_named_stream(dv, monkeypatch, as_handle):
    s = serving(np.random.default_rng(4))
    x, w = s["x"].float(), s["gain"].float()

    def every_call(**kw):
        out, total, rstd = dv.rms_norm(x, w, residual=x, want_rstd=True, **kw)
        got = [out, total, rstd, *dv.rms_norm_backward(x, total, w, rstd, **kw)]
        got += dv.rms_norm_f8(x, w, residual=x, **kw)
        q, sc, tq, ts = dv.quantize_f8(x, want_columns=True, **kw)
        got += [q, sc, tq, ts, dv.product_f8(q, sc, q, sc, tile=1, **kw), dv.product_f8(tq, ts, tq, ts, tile=1, **kw)]
        got.append(dv.adjust_logits(x, bias_ids=s["bias_ids"], bias=s["bias"], **kw))
        return [t.view(torch.uint8) if t.dtype == dv.F8 else t for t in got]

    want = every_call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    at, empty = [], torch.empty

    def recorded(*a, **k):
        at.append(torch.cuda.current_stream(DEV).cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(torch, "empty", recorded)
    got = every_call(stream=side.cuda_stream if as_handle else side)
    monkeypatch.undo()
    side.synchronize()
    assert len(at) >= len(got) and set(at) == {side.cuda_stream}
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_two_steps_at_once(dv):
    """Decode steps on two streams, each with its own arrays: results are those of one after the other."""
    sets = [serving(np.random.default_rng(k), B=40, V=20011) for k in (5, 6)]
    heads = [dv.quantize_f8(s["head"], tile=128)[:2] for s in sets]
    want = [decode(dv, s, *h, True) for s, h in zip(sets, heads)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(5):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[k].append(decode(dv, sets[k], *heads[k], True))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            for a, b in zip(g, want[k]):
                assert torch.equal(a, b)


def test_autograd_of_the_norm(dv):
    from paper_2403_06988_amd import autograd as dva
    rng = np.random.default_rng(7)
    t = lambda *shape: torch.from_numpy(rng.normal(size=shape)).float().to(DEV)  # noqa: E731
    x, res, w, g, gt = t(30, 77), t(30, 77), t(77), t(30, 77), t(30, 77)
    leaves = [v.clone().requires_grad_() for v in (x, res, w)]
    out, total = dva.rms_norm(leaves[0], leaves[2], 1e-5, leaves[1])
    ((out * g).sum() + (total * gt).sum()).backward()
    _, h, r = dv.rms_norm(x, w, 1e-5, residual=res, want_rstd=True)
    dx, dx_tol, dw, dw_tol = norm_backward_reference(g.cpu(), h.cpu(), w.cpu(), r.cpu(), gt.cpu())
    check(leaves[0].grad, dx, dx_tol, "x")
    check(leaves[1].grad, dx, dx_tol, "residual")
    check(leaves[2].grad, dw, dw_tol, "weight")
    # without a residual; only one of the results used; only one input wants a gradient
    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    (dva.rms_norm(a, b, 1e-5) * g).sum().backward()
    _, _, r = dv.rms_norm(x, w, 1e-5, want_rstd=True)
    dx, dx_tol, dw, dw_tol = norm_backward_reference(g.cpu(), x.cpu(), w.cpu(), r.cpu(), None)
    check(a.grad, dx, dx_tol, "x alone")
    check(b.grad, dw, dw_tol, "weight alone")
    a = x.clone().requires_grad_()
    (dva.rms_norm(a, w, 1e-5, res)[1] * gt).sum().backward()
    assert torch.equal(a.grad, gt)
    b = w.clone().requires_grad_()
    (dva.rms_norm(x, b, 1e-5, res)[0] * g).sum().backward()
    assert b.grad is not None
    a = x.clone().requires_grad_()
    (first,) = torch.autograd.grad((dva.rms_norm(a, w) ** 2).sum(), a, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(first.sum(), a)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_autograd_of_the_8_bit_product(dv, dtype):
    """Result and gradients against 64-bit products of what the quantized operands stand for."""
    from paper_2403_06988_amd import autograd as dva
    rng = np.random.default_rng(8)
    N, D, V = 150, 200, 333
    x, w, g = (torch.from_numpy(rng.normal(size=s)).to(dtype) for s in ((N, D), (V, D), (N, V)))
    a, b = x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_()
    out = dva.linear_f8(a, b)
    out.backward(g.to(DEV))
    xq, wq = quantize(x, 1), quantize(w, 128)
    wt = quantize(w.t().contiguous(), 128)
    gq, gt, xt = quantize(g, 1), quantize(g.t().contiguous(), 1), quantize(x.t().contiguous(), 1)
    check(out, *product_reference(*xq, *wq, 128, dtype), "result")
    check(a.grad, *product_reference(*gq, *wt, 128, dtype), "x")
    check(b.grad, *product_reference(*gt, *xt, 1, dtype), "weight")
    # and near what it stands for: 8-bit operands are off by 2^-4 of a term at most
    exact = g.double() @ w.double()
    size = g.double().abs() @ w.double().abs()
    assert ((a.grad.cpu().double() - exact).abs() <= 0.14 * size).all()
    assert values(*xq, 1).shape == (N, 256)
    only = x.to(DEV).requires_grad_()
    dva.linear_f8(only, w.to(DEV)).backward(g.to(DEV))
    assert torch.equal(only.grad, a.grad)
    only = w.to(DEV).requires_grad_()
    dva.linear_f8(x.to(DEV), only).backward(g.to(DEV))
    assert torch.equal(only.grad, b.grad)
    none, only = x[:0].to(DEV).requires_grad_(), w.to(DEV).requires_grad_()
    dva.linear_f8(none, only).sum().backward()
    assert none.grad.shape == (0, D) and (only.grad == 0).all()
