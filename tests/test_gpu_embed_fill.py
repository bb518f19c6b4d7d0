"""The table's gradient for tables that the sort does not cover: rows that no
token names are zeros everywhere, whatever the alignment and the runs of absent tokens."""
import numpy as np
import pytest
import torch

from tests.test_gpu_embed import DEV, strided, tokens
from tests.train_common import check, embed_backward_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2403_06988_amd as dv_mod
    return dv_mod


# tables of 60 to 210 MB; odd widths, rows longer than what a wave fills at once
@pytest.mark.parametrize("N,D,V,how,dtype", [
    (1, 1024, 40000, "one", torch.bfloat16), (5, 1111, 30011, "any", torch.bfloat16), (300, 1501, 20000, "frequent", torch.float32),
    (1000, 4096, 10003, "frequent", torch.bfloat16), (3000, 1024, 50021, "any", torch.bfloat16), (64, 40000, 701, "few", torch.float32),
    (8192, 1031, 50000, "any", torch.float32), (8192, 2048, 50001, "frequent", torch.bfloat16),
])
def test_rows_that_no_token_names(dv, N, D, V, how, dtype):
    print(f"embed fill N={N} D={D} V={V} {how} {dtype}", flush=True)
    rng = np.random.default_rng(N + D)
    g = torch.from_numpy(rng.standard_normal((N, D), dtype=np.float32)).to(dtype)
    ids = tokens(rng, N, V, how)
    if N > 4:
        ids[0], ids[1] = V - 1, 0
    room = torch.full((V * D + 3,), float("nan"), dtype=dtype, device=DEV)
    for off, pad in ((0, 0), (3, 5)):
        room.fill_(float("nan"))
        out = room[off:off + V * D].view(V, D)
        got = dv.embed_backward(strided(g, pad), ids.to(DEV), V, 0.5, grad_weight=out)
        torch.cuda.synchronize()
        named = torch.unique(ids[(ids >= 0) & (ids < V)].long())
        rest = torch.ones(V, dtype=torch.bool, device=DEV)
        rest[named.to(DEV)] = False
        assert bool((got[rest] == 0).all())
        at = torch.searchsorted(named, ids.long().clamp(0, V - 1)).int()
        at[(ids < 0) | (ids >= V)] = -1
        want, tol = embed_backward_reference(g, at, len(named), 0.5)
        check(got[named.to(DEV)], want, tol, "grad_weight")
        assert bool(torch.isnan(room[:off]).all()) and bool(torch.isnan(room[off + V * D:]).all())
