"""The training operators together: as differentiable functions against
float64 autograd, a tied table's accumulated gradient, and the example's training."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from tests.train_common import masks, pack_mask, row_mask

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def test_differentiable_functions_match_float64_autograd(dv):
    """embed -> mix -> head loss, and -> logits -> distillation, one shared
    table: the fp32 gradients against torch's in float64 on the CPU.  Bound: the
    operators' fp32 sums (at most 300 terms) and the two torch products between
    them, 2^-24 a term, with room for the chain: 1e-4 of the largest element."""
    from paper_2403_06988_amd import autograd as dva
    rng = np.random.default_rng(4)
    N, D, V, K = 40, 32, 300, 8
    table = torch.from_numpy(rng.normal(size=(V, D)) * 0.5)
    mix = torch.from_numpy(rng.normal(size=(D, D)) * 0.3)
    ids = torch.from_numpy(rng.integers(-1, V, N).astype(np.int32))
    may = masks(rng, 3, V, (0.3, 1.0))
    states = torch.from_numpy(rng.integers(-1, 3, N).astype(np.int32))
    mask = row_mask(may, states, N, V)
    targets = torch.from_numpy(rng.integers(0, V, N).astype(np.int32))
    t_ids = torch.from_numpy(rng.integers(0, V, (N, K)).astype(np.int32))
    t_top = torch.from_numpy(rng.normal(size=(N, K)) * 2).float()

    def forward(table, mix, own):
        if own:
            al, st = pack_mask(may).to(DEV), states.to(DEV)
            x = dva.embed(table, ids.to(DEV), 1.5) @ mix
            a = dva.head_loss(x, table, targets.to(DEV), al, st)
            b = dva.distill_loss(x @ table.t(), t_ids.to(DEV), t_top.to(DEV), 0.8, al, st)
            return (a.sum() + 0.5 * b.sum()) / N
        x = torch.where((ids >= 0)[:, None], table[ids.clamp(min=0).long()] * 1.5, torch.zeros((), dtype=torch.float64)) @ mix
        z = x @ table.t()
        zm = z.masked_fill(~mask, -1e300)
        live = mask.any(1)
        part = live & mask[torch.arange(N), targets.long()]
        a = torch.where(part, torch.logsumexp(zm, 1) - z[torch.arange(N), targets.long()], torch.zeros(()).double())
        total = a.sum()
        for n in range(N):
            at = t_ids[n].long()
            keep = mask[n, at]
            if not live[n] or not keep.any():
                continue
            lq = torch.log_softmax(0.8 * t_top[n].double()[keep], 0)
            lp = torch.log_softmax(0.8 * zm[n], 0)[at[keep]]
            total = total + 0.5 * (lq.exp() * (lq - lp)).sum()
        return total / N

    t64, m64 = table.clone().requires_grad_(), mix.clone().requires_grad_()
    want = forward(t64, m64, False)
    want.backward()
    t32, m32 = table.float().to(DEV).requires_grad_(), mix.float().to(DEV).requires_grad_()
    got = forward(t32, m32, True)
    got.backward()
    assert abs(got.item() - want.item()) < 1e-5 * abs(want.item())
    for a, b in ((t32.grad, t64.grad), (m32.grad, m64.grad)):
        assert (a.cpu().double() - b).abs().max() < 1e-4 * b.abs().max()


def test_frozen_inputs_get_no_gradient(dv):
    from paper_2403_06988_amd import autograd as dva
    x = torch.randn(10, 64, device=DEV).bfloat16().requires_grad_()
    w = torch.randn(100, 64, device=DEV).bfloat16()
    t = torch.arange(10, dtype=torch.int32, device=DEV)
    dva.head_loss(x, w, t).mean().backward()
    assert x.grad is not None and x.grad.dtype == torch.bfloat16 and w.grad is None


def test_example_learns(dv):
    spec = importlib.util.spec_from_file_location("train_proposer", os.path.join(ROOT, "examples", "train_proposer.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    r = mod.main(steps=80, verbose=False)
    assert np.mean(r["token_loss"][-5:]) < 0.8 * np.mean(r["token_loss"][:5])
    assert np.mean(r["distill_loss"][-5:]) < 0.5 * np.mean(r["distill_loss"][:5])
    assert r["after"] > r["before"]
