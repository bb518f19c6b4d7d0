"""Calls from the last layer to the logits that are refused (no GPU needed)."""
import pytest
import torch

import paper_2403_06988_amd as dv
from paper_2403_06988_amd import autograd as dva


@pytest.mark.parametrize("x,w", [((4, 100), (30, 120)), ((4, 100), (30, 128)), ((4, 128), (30, 100)), ((4, 256), (30, 128)),
                                 ((100,), (30, 100)), ((4, 100), (100,))])
def test_linear_f8_refuses_other_depths(x, w):
    """Operands are padded to whole blocks of 128: rows of 100 and 120 would both be 128 long."""
    with pytest.raises(ValueError, match="weight must be"):
        dva.linear_f8(torch.zeros(x), torch.zeros(w))


def product(M, N, K, ws, nb):
    """The call with fake pointers, its result where its workspace is: refused as overlapping, past the workspace's checks."""
    P, GB = 0x7F0000000000, 1 << 30
    return dv.lib.dv_product_f8(P, K, P + 200 * GB, P + 20 * GB, K, P + 300 * GB, 128, M, N, K, dv.DV_BF16, ws, N, ws, nb, None)


@pytest.mark.parametrize("N,K", [(32000, 4096), (1024, 8192), (1, 128), (257, 1 << 17), (4096, 32000), (128256, 1024)])
def test_a_products_workspace_for_every_smaller_batch(N, K):
    """One size serves calls of up to as many rows, and never falls; that of a call's own rows may."""
    up_to, own = dv.product_f8_workspace_bytes_up_to, dv.product_f8_workspace_bytes
    rows = sorted({r for c in (1, 16, 32, 64, 128, 192, 256, 512, 640, 1000, 1024, 2048, 4096, 5000) for r in (c - 1, c, c + 1)})
    most, sizes = 0, []
    for r in rows:
        most = max(most, own(r, N, K))
        sizes.append(up_to(r, N, K))
        assert sizes[-1] >= most
    assert sizes == sorted(sizes)
    for r in rows[1:]:
        if own(r, N, K):
            assert product(r, N, K, 0x7F0000000000 + (100 << 30), sizes[-1]) == 4     # DV_ERR_ALIAS: the workspace is enough
    if (N, K) == (32000, 4096):
        assert own(64, N, K) > own(65, N, K)


def test_a_products_workspace_up_to_every_row():
    """Row by row where the plan changes often."""
    for N, K in ((130, 6016), (1024, 8192), (4096, 2048)):
        most = last = 0
        for r in range(0, 1400):
            most = max(most, dv.product_f8_workspace_bytes(r, N, K))
            now = dv.product_f8_workspace_bytes_up_to(r, N, K)
            assert now >= most and now >= last
            last = now


def test_workspace_up_to_outside_the_limits():
    q = dv.product_f8_workspace_bytes_up_to
    assert q(-1, 8, 128) == q(8, 0, 128) == q(8, 8, 100) == q(8, 8, 0) == q(1 << 20, 1 << 16, 128) == 0


def test_exact_sums_of_no_other_type():
    """The choice stands beside a type; other bits are refused as types are."""
    P, GB = 0x7F0000000000, 1 << 30
    call = lambda dt: dv.lib.dv_product_f8(P, 256, P + GB, P + 2 * GB, 256, P + 3 * GB, 128, 8, 300, 256, dt, P + 16, 300,  # noqa: E731
                                           P + 5 * GB, 1 << 50, None)
    assert call(dv.DV_BF16 | dv.DV_EXACT_SUMS) == call(dv.DV_F32 | dv.DV_EXACT_SUMS) == 4      # as far as the overlap
    for dt in (2 | dv.DV_EXACT_SUMS, 2 * dv.DV_EXACT_SUMS, -1, dv.DV_EXACT_SUMS << 1 | dv.DV_BF16):
        assert call(dt) == 3                                                                    # DV_ERR_DTYPE


P, GB = 0x7F0000000000, 1 << 30


def norm(rstd=P + 5 * GB):
    return dv.lib.dv_rms_norm(P, 64, P + GB, 64, P + 2 * GB, 1, 8, 64, 1e-6, P + 2 * GB, P + 4 * GB, rstd, None, None, None)


def norm_back(rstd=P + 3 * GB):
    return dv.lib.dv_rms_norm_backward(P, 64, P + GB, 64, P + 2 * GB, rstd, None, 64, 1, 8, 64, P + 5 * GB, P + 5 * GB, P + 7 * GB,
                                       1 << 40, None)


def adjust(history=P + GB, lengths=P + 2 * GB, prompts=P + 3 * GB, repetition=P + 4 * GB, presence=P + 5 * GB, frequency=P + 6 * GB,
           ids=P + 7 * GB, bias=P + 8 * GB, allow=P + 9 * GB, states=P + 10 * GB):
    return dv.lib.dv_adjust_logits(P, 1000, 1, 8, 1000, history, 50, 50, lengths, prompts, repetition, presence, frequency, ids, bias, 4,
                                   allow, 2, states, P + 2, 1000, None)


@pytest.mark.parametrize("call,names", [(norm, ["rstd"]), (norm_back, ["rstd"]),
                                        (adjust, ["history", "lengths", "prompts", "repetition", "presence", "frequency", "ids", "bias",
                                                  "allow", "states"])])
def test_arrays_of_four_bytes_off_their_alignment(call, names):
    """fp32 and int32 arrays as the others (calls that a later check, the overlap's, would stop)."""
    assert call() == 4                                              # DV_ERR_ALIAS
    for name in names:
        place = call.__defaults__[call.__code__.co_varnames.index(name)]
        for off in (1, 2):
            assert call(**{name: place + off}) == 1                 # DV_ERR_INVALID_ARG
            assert b"aligned" in dv.lib.dv_last_error()
