"""Attention over latents where most sequences are short and one is long, under tables so wide that
the work is split evenly.  Oracles and tolerances are those of the operators' own tests."""

import numpy as np
import pytest
import torch

from test_gpu_latent_attention import Case
from test_gpu_latent_prompt import Prompt

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,batch", [(20, 700), (40, 530), (100, 515), (3, 2100)])
def test_one_long_sequence_among_many(heads, batch, fp8):
    rng = np.random.default_rng(heads)
    lens = rng.integers(0, 60, batch)
    lens[batch // 3] = 1230  # a table of 79 pages
    Case(lens, heads, 1, 256, fp8, seed=heads).check()


def test_a_workspace_for_the_widest_serves_narrower_and_fewer():
    import paper_2609_36899_amd as P
    ws = torch.full((P.paged_latent_attention_workspace_bytes(P.BF16, 700, 2, 20, 256, 79),), 0xFF,
                    dtype=torch.uint8, device="cuda")
    rng = np.random.default_rng(5)
    for batch, n_q, top in ((700, 2, 1200), (700, 1, 300), (511, 1, 1000), (40, 2, 1200)):
        lens = rng.integers(0, 50, batch)
        lens[3] = top
        case = Case(lens, 20, n_q, 256, False, seed=batch)
        case.check(case.run(workspace=ws))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,rows,keys", [
    (20, [64] * 40, [64] * 39 + [2564]), (20, [64] * 40, [2564] + [64] * 39),
    (8, [3] * 100, [3] * 50 + [4003] + [3] * 49), (130, [32] * 17, [40] * 16 + [3000])])
def test_one_long_context_among_fresh_prompts(heads, rows, keys, dim):
    Prompt(rows, keys, heads, dim, seed=heads).check()
