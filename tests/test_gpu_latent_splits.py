"""Where the work of latent and prompt attention is cut, and copies of very large pages: sizes
on both sides of each rule that chooses a split.  Oracles and tolerances are those of the
operators' own tests."""

import numpy as np
import pytest
import torch

from test_gpu_latent_attention import Case
from test_gpu_latent_prompt import Prompt

pytestmark = pytest.mark.gpu


def _P():
    import paper_2609_36899_amd as P
    return P


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("latent", [256, 512])
def test_pieces_of_many_lengths(latent, fp8):
    # Units of 1 to 40 tiles and empty ones among them: pieces that begin, go on and end anywhere,
    # and groups whose stretch ends ahead of a unit's first tile.
    rng = np.random.default_rng(latent + fp8)
    lens = np.concatenate([rng.integers(0, 4, 9), rng.integers(1, 1300, 30), [0, 1, 16, 17, 2500]])
    rng.shuffle(lens)
    for heads, n_q in ((16, 1), (5, 3), (20, 1), (33, 1), (100, 1)):
        Case(lens, heads, n_q, latent, fp8, seed=heads).check()


@pytest.mark.parametrize("batch", [511, 512, 700])
def test_few_rows_of_many_sequences(batch):
    # Stretches up to 2047 units of one row tile.
    lens = np.random.default_rng(batch).integers(0, 40, batch)
    lens[7] = 600
    Case(lens, 3, 1, 256, True, seed=batch).check()


def test_more_units_than_stretches_take():
    lens = np.random.default_rng(0).integers(0, 20, 2050)
    lens[100] = 300
    Case(lens, 2, 1, 256, False, seed=1).check()


def test_wide_blocks_of_many_sequences():
    lens = np.random.default_rng(1).integers(0, 40, 520)
    lens[3] = 300
    Case(lens, 20, 1, 256, True, seed=2).check()


@pytest.mark.parametrize("rows,keys", [
    ([1024] * 4, [1024] * 4),            # 36 x 32 blocks of all heads: a group each
    ([128] * 4, [700] * 4),              # behind contexts: equal stretches
    ([128] * 20, [400, 128] * 10)])
def test_blocks_and_stretches_of_prompts(rows, keys):
    Prompt(rows, keys, 32, 64, seed=len(rows)).check()


def test_pages_of_more_parts_than_a_grid_takes():
    # Copied byte by byte, 512 a group.
    n = 65535 * 512 + 777
    pool = torch.empty((3, n), dtype=torch.uint8, device="cuda")
    for i in range(3):
        pool[i] = (torch.arange(n, device="cuda") * (i + 3) % 251).to(torch.uint8)
    want = pool[2].clone()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    before = pool[1].clone()
    _P().paged_copy_pages(pool, i32([2]), i32([0]))
    assert torch.equal(pool[0], want) and torch.equal(pool[1], before) and torch.equal(pool[2], want)
