"""Attention over latents where what is not seen is not finite: pages that are not there between
others that are, and drafted tokens.  Oracle and tolerances are those of
test_gpu_latent_attention.py."""

import numpy as np
import pytest
import torch

from test_gpu_latent_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads", [3, 16, 20, 64, 128])
def test_page_0_is_no_stand_in_for_pages_that_are_not_there(heads, latent, fp8):
    """Its latents, keys and scales are NaN throughout, and no table names it."""
    case = Case([700, 65, 16, 330], heads, latent=latent, fp8=fp8, seed=31)
    spare = int(np.setdiff1d(np.arange(case.P), np.concatenate(
        [case.table[b, :-(-int(n) // 16)] for b, n in enumerate(case.lens)]))[0])
    # Page 0's tokens move to the page that no sequence has.
    case.k[spare] = case.k[0]
    if fp8:
        case.codes[spare], case.ts[spare] = case.codes[0], case.ts[0]
    else:
        case.c[spare] = case.c[0]
    case.table[case.table == 0] = spare
    case.spoil(0, 0)
    for b, at in ((0, [1, 2, 9, 20, 33, 43]), (1, [0, 4]), (2, [0]), (3, list(range(3, 17)))):
        for i, page in enumerate(at):
            case.table[b, page] = (-1, case.P, 1 << 30, -(1 << 31))[i % 4]
    case.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), 2.0 ** 100])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads,n_q", [(3, 5), (8, 4), (32, 4), (100, 3)])
def test_scales_of_later_tokens_reach_no_earlier_ones(heads, n_q, latent, bad):
    """A drafted token whose scale is not finite, or as large as one may be, its codes being so."""
    case = Case([70, 64, 200], heads, n_q, latent=latent, fp8=True, seed=32)
    want, tol = case.expected()
    for b, n in enumerate(case.lens):
        p = n - n_q + 2  # the third of them
        case.ts[case.table[b, p // 16], p % 16] = bad
    got = case.run().double().cpu().numpy()
    assert (np.abs(got[:, :2] - want[:, :2]) <= tol[:, :2]).all()
    if not np.isfinite(bad):
        assert not np.isfinite(got[:, 2:]).all(-1).any()


@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads,n_q", [(5, 1), (16, 1), (40, 1), (128, 1), (32, 4)])
def test_scales_that_are_no_powers_of_two(heads, n_q, latent):
    Case([77, 300, 1], heads, n_q, latent=latent, fp8=True, pow2=False, seed=33).check()
