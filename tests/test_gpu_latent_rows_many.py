"""paged_latent_rows of more rows than caches hold, ragged and with remainders of every size that a
wave and a work group have, equal to a gather."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ROPE = 64


def _i32(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("R,many", [(512, 65536), (256, 117964)])
def test_many_rows(R, many, fp8):
    import paper_2609_36899_amd as P
    rng = np.random.default_rng(R + fp8)
    pool = 300
    if fp8:
        raw = rng.integers(0, 256, (pool, 16, R + 2 * ROPE)).astype(np.uint8)
        codes = raw[..., :R]
        codes[(codes & 0x7F) == 0x7F] = 0x38  # no NaN, so that values compare
        pages = torch.from_numpy(raw).cuda()
        # Powers of two: what reads back is a bf16 number.
        scales = torch.exp2(_i32(rng.integers(-9, 9, (pool, 16))).float())
        values = pages[..., :R].view(torch.float8_e4m3fn).float() * scales[..., None]
        keys = pages[..., R:].contiguous().view(torch.int16)
    else:
        pages = torch.from_numpy(rng.standard_normal((pool, 16, R + ROPE)).astype(np.float32))
        pages, scales = pages.to(torch.bfloat16).cuda(), None
        values, keys = pages[..., :R].float(), pages[..., R:].contiguous().view(torch.int16)
    for n in (many // 2 - 7, many - 3, many, many + 1, many + 1003):
        # Ragged sequences, some of them empty, a part of each of the others; ahead of, and
        # behind them rows of none; places without a page.
        held = np.concatenate([[0, 1, 5, 0, 37], rng.multinomial(n - 43 - 9, np.ones(11) / 11)])
        starts = 4 + np.concatenate([[0], np.cumsum(held)])
        lens = held + rng.integers(0, 50, len(held))
        stride = int(lens.max()) // 16 + 1
        table = rng.integers(0, pool, (len(held), stride)).astype(np.int32)
        table[rng.random(table.shape) < 0.02] = -1
        c = torch.full((n, R), 7.0, dtype=torch.bfloat16, device="cuda")
        k = torch.full((n, ROPE), 7.0, dtype=torch.bfloat16, device="cuda")
        P.paged_latent_rows(pages, _i32(lens), _i32(starts), _i32(table), c, k, scales=scales)
        seq = np.repeat(np.arange(len(held)), held)
        pos = (lens - starts[1:])[seq] + np.arange(starts[0], starts[-1])
        page = table[seq, pos // 16]
        row = np.arange(starts[0], starts[-1])[page >= 0]
        at = torch.from_numpy(page[page >= 0].astype(np.int64)).cuda()
        slot = torch.from_numpy((pos % 16)[page >= 0]).cuda()
        want_c, want_k = torch.full_like(c, 7.0), torch.full_like(k, 7.0)
        row = torch.from_numpy(row).cuda()
        want_c[row] = values[at, slot].to(torch.bfloat16)
        want_k[row] = keys[at, slot].view(torch.bfloat16)
        assert torch.equal(c, want_c)
        assert torch.equal(k.view(torch.int16), want_k.view(torch.int16))
