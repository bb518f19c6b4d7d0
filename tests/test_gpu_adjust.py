"""Adjusted logits against the definition in 64 bits: histories, prompts,
penalties, biases, masks, in place and not."""
import math

import numpy as np
import pytest
import torch

from tests.logits_common import adjust_reference
from tests.train_common import check, masks, pack_mask, row_mask

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


def requests(rng, B, V, H, nb, S):
    """(arguments on the CPU, mask [B][V] or None)."""
    f = lambda a: torch.from_numpy(np.asarray(a, np.float32))  # noqa: E731
    i = lambda a: torch.from_numpy(np.asarray(a, np.int32))  # noqa: E731
    how = {}
    if H is not None:
        hist = np.minimum(V ** rng.random((B, H)) - 1, V - 1).astype(np.int64)
        hist = np.where(rng.random((B, H)) < 0.05, rng.integers(-3, V + 3, (B, H)), hist)   # some outside
        lengths = rng.integers(0, H + 1, B)
        lengths[0] = H + 5                          # clamped
        if B > 2:
            lengths[1], lengths[2] = 0, -4
        how.update(history=i(hist), lengths=i(lengths), prompts=i(rng.integers(-1, H + 2, B)),
                   repetition=f(1 + rng.random(B)), presence=f(rng.normal(size=B)), frequency=f(rng.random(B)))
    if nb is not None:
        ids = rng.integers(-2, V + 2, (B, nb))
        if nb > 3:
            ids[:, nb - 1] = ids[:, 0]
            ids[:, nb // 2] = ids[:, 0]
            if H:
                ids[:, 1] = how["history"][:, 0].numpy()
        how.update(bias_ids=i(ids), bias=f(rng.normal(size=(B, nb)) * 5))
    may = None
    if S:
        may_s = masks(rng, S, V, [0.0, 0.5, 1.0, 0.02])
        states = rng.integers(-1, S + 1, B).astype(np.int32)
        how.update(allow=pack_mask(may_s), states=torch.from_numpy(states))
        may = row_mask(may_s, states, B, V)
    return how, may


def device_args(how):
    d = {k: v.to(DEV) for k, v in how.items()}
    if "prompts" in d:
        d["prompt_lengths"] = d.pop("prompts")
    return d


def reference(z, how, may):
    return adjust_reference(z, **{k: v for k, v in how.items() if k not in ("allow", "states")}, may=may)


def compare(got, z, want, tol, kept, may):
    got = got.cpu()
    check(got, want, tol, "logits")
    bits = torch.int16 if z.dtype == BF else torch.int32
    if may is not None:
        kept = kept & may
    assert torch.equal(got.view(bits)[kept], z.view(bits)[kept])       # copied, not computed


CASES = [(1, 1, 1, 1, 0), (1, 1000, 0, 0, 3), (3, 31, 5, 2, 2), (5, 8192, 64, 4, 0), (4, 8193, 300, None, 5),
         (7, 20011, None, 33, 0), (6, 50257, 3000, 300, 0), (3, 128256, 700, 8, 4), (2, 16385, 20000, 1024, 3),
         (9, 4099, None, None, 6), (230, 20011, 50, 9, 4), (260, 16500, 2500, None, 0)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,V,H,nb,S", CASES)
def test_adjusted_logits(dv, B, V, H, nb, S, dtype):
    rng = np.random.default_rng(B * 1009 + V)
    z = torch.from_numpy(rng.normal(size=(B, V)) * 4).to(dtype)
    how, may = requests(rng, B, V, H, nb, S)
    want, tol, kept = reference(z, how, may)
    pad = 3 if V % 8 else 0
    buf = torch.full((B * (V + pad) + 1,), 77.0, dtype=dtype, device=DEV)
    x = buf[1:].view(B, V + pad)[:, :V]
    x.copy_(z)
    args = device_args(how)
    got = dv.adjust_logits(x, **args)
    compare(got, z, want, tol, kept, may)
    assert torch.equal(x.cpu(), z)
    wide = torch.full((B, V + 4), 5.0, dtype=dtype, device=DEV)
    dv.adjust_logits(x, **args, out=wide[:, 1:V + 1])
    assert torch.equal(wide[:, 1:V + 1], got) and (wide[:, 0] == 5).all() and (wide[:, V + 1:] == 5).all()
    dv.adjust_logits(x, **args, out=x)
    assert torch.equal(x, got)
    if pad:
        assert (buf[1:].view(B, V + pad)[:, V:] == 77).all() and buf[0] == 77


@pytest.mark.parametrize("absent", ["prompts", "repetition", "presence", "frequency"])
def test_each_penalty_may_be_absent(dv, absent):
    rng = np.random.default_rng(3)
    z = torch.from_numpy(rng.normal(size=(4, 3000))).float()
    how, _ = requests(rng, 4, 3000, 200, None, 0)
    del how[absent]
    want, tol, kept = reference(z, how, None)
    compare(dv.adjust_logits(z.to(DEV), **device_args(how)), z, want, tol, kept, None)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("mask", [False, True])
def test_special_values(dv, dtype, in_place, mask):
    """Infinities, NaN and the type's extremes among the logits, named or not, allowed or not."""
    rng = np.random.default_rng(8)
    B, V = 6, 9000
    top = torch.finfo(dtype).max
    z = torch.from_numpy(rng.normal(size=(B, V))).to(dtype)
    for k, v in enumerate((math.inf, -math.inf, math.nan, top, -top, 0.0, -0.0)):
        z[:, k * 17:k * 17 + 9] = v
    how, may = requests(rng, B, V, 40, 12, 5 if mask else 0)
    how["history"][:, :20] = torch.arange(20, dtype=torch.int32) * 7
    how["lengths"][:] = 40
    want, tol, kept = reference(z, how, may)
    if dtype == BF:    # what rounds beyond the type's largest
        want = want.to(F32).to(BF).double()
    else:
        want = want.to(F32).double()
    x = z.to(DEV)
    got = dv.adjust_logits(x, **device_args(how), out=x if in_place else None).cpu()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan)
    check(torch.where(nan, torch.zeros((), dtype=dtype), got), torch.where(nan, torch.zeros(()).double(), want),
          torch.where(nan, torch.zeros(()).double(), tol * 2), "values")
    bits = torch.int16 if dtype == BF else torch.int32
    kept = kept if may is None else kept & may
    assert torch.equal(got.view(bits)[kept], z.view(bits)[kept])


def test_bans_and_forced_tokens(dv):
    """-inf as a bias bans a token; a state that allows nothing leaves -inf everywhere."""
    z = torch.zeros((2, 100), device=DEV)
    ids = torch.tensor([[3, 4], [3, -1]], dtype=torch.int32, device=DEV)
    bias = torch.tensor([[-math.inf, 2.0], [-math.inf, 9.0]], device=DEV)
    out = dv.adjust_logits(z, bias_ids=ids, bias=bias).cpu()
    assert out[0, 3] == out[1, 3] == -math.inf and out[0, 4] == 2 and out[1, 4] == 0 and (out[:, 5:] == 0).all()
    allow = torch.zeros((1, 4), dtype=torch.int32, device=DEV)
    out = dv.adjust_logits(z, allow=allow, states=torch.tensor([0, -1], dtype=torch.int32, device=DEV))
    assert (out == -math.inf).all()


def test_no_rows(dv):
    z = torch.empty((0, 50), device=DEV)
    assert dv.adjust_logits(z).shape == (0, 50)
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    assert dv.adjust_logits(z, history=torch.empty((0, 9), dtype=torch.int32, device=DEV), lengths=none).shape == (0, 50)
