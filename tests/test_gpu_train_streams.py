"""The training calls on a stream named by the caller: what they allocate
belongs to that stream, results are those of the current one; and gradients of
gradients raise."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def inputs(N=150, D=72, V=3001, K=7):
    rng = np.random.default_rng(5)
    f32 = lambda *shape: torch.from_numpy(rng.normal(size=shape)).float().to(DEV)
    ids = torch.from_numpy(rng.integers(-1, V, N).astype(np.int32)).to(DEV)
    top_ids = torch.from_numpy(rng.integers(0, V, (N, K)).astype(np.int32)).to(DEV)
    return f32(V, D), ids, f32(N, D), f32(N), f32(N, V), top_ids, f32(N, K)


def every_call(dv, table, ids, x, g, z, top_ids, top, stream):
    kw = dict(stream=stream)
    loss, lse = dv.head_loss(x, table, ids, **kw)
    out = [loss, lse, *dv.head_loss_backward(x, table, ids, lse, g, **kw)]
    out.append(dv.distill_loss(z, top_ids, top, **kw))
    out += dv.distill_loss_backward(z, top_ids, top, g, **kw)
    out.append(dv.embed(table, ids, 2.0, **kw))
    out.append(dv.embed_backward(x, ids, table.shape[0], 2.0, **kw))
    return out


@pytest.mark.parametrize("as_handle", [False, True])
def test_arrays_come_from_the_named_stream(dv, monkeypatch, as_handle):
    args = inputs()
    want = every_call(dv, *args, stream=None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    at = []
    empty = torch.empty

    def recorded(*a, **k):
        at.append(torch.cuda.current_stream(DEV).cuda_stream)
        return empty(*a, **k)

    monkeypatch.setattr(torch, "empty", recorded)
    got = every_call(dv, *args, stream=side.cuda_stream if as_handle else side)
    monkeypatch.undo()
    side.synchronize()
    assert len(at) >= len(got) and set(at) == {side.cuda_stream}
    assert torch.cuda.current_stream(DEV).cuda_stream != side.cuda_stream
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_gradients_of_gradients_raise(dv):
    from paper_2403_06988_amd import autograd as dva
    table, ids, x, g, z, top_ids, top = inputs()
    for value, leaf in ((lambda t: (dva.embed(t, ids) ** 2).sum(), table), (lambda t: (dva.head_loss(t, table, ids) ** 2).sum(), x),
                        (lambda t: (dva.distill_loss(t, top_ids, top) ** 2).sum(), z)):
        leaf = leaf.clone().requires_grad_()
        (first,) = torch.autograd.grad(value(leaf), leaf, create_graph=True)
        with pytest.raises(RuntimeError):
            torch.autograd.grad(first.sum(), leaf)
