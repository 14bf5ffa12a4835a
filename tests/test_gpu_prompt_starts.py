"""latent_prompt_attention on starts that no prompts have: what descends is nothing, and a call
that is nothing writes nothing."""

import numpy as np
import pytest
import torch

from test_gpu_latent_prompt import Prompt

pytestmark = pytest.mark.gpu


def _i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.parametrize("heads", [2, 200])  # equal stretches, and a group a block
@pytest.mark.parametrize("starts", [[5, 2, 300], [0, 300, 299], [300, 0, 0], [0, 300, -1], [1 << 30, 0, 300]])
def test_rows_that_descend(starts, heads):
    case = Prompt([200, 100], [230, 100], heads, 64, seed=1)
    assert (case.run(q_start=_i32(starts)) == 7.0).all()


@pytest.mark.parametrize("seqs", [100, 1000, 1500])
def test_sequences_that_share_their_rows(seqs):
    """Every second sequence holds all rows: more tiles in all than the rows and keys allow."""
    case = Prompt([4000], [9000], 1, 64, seed=2)
    q = np.tile([0, 4000], seqs // 2 + 1)[:seqs + 1]
    k = np.tile([0, 9000], seqs // 2 + 1)[:seqs + 1]
    assert (case.run(q_start=_i32(q), k_start=_i32(k)) == 7.0).all()


def test_keys_that_descend():
    """Such a sequence has none, and its rows are zeros; the others are as ever."""
    case = Prompt([70, 40, 90], [100, 60, 120], 3, 128, seed=3)
    case.ks = np.array([0, 100, 90, 210], np.int32)
    got = case.run()
    assert (got[70:110] == 0).all()
    want, tol = case.expected()
    got = got.double().cpu().numpy()
    ok = np.r_[0:70, 110:200]
    assert (np.abs(got - want) <= tol)[ok].all()
