"""Which calls of latent and prompt attention split their work over groups alike, as the library's
workspaces tell: partials are what such a split leaves.  No launch is made."""

import pytest

from paper_2609_36899_amd import _native as N
from test_latent_refusals import _attn, _prompt, _ws


@pytest.mark.parametrize("kv", [N.BF16, N.FP8_E4M3])
@pytest.mark.parametrize("heads,batch", [(16, 2048), (16, 4095), (32, 512), (32, 1000), (64, 4095),
                                         (128, 512), (128, 3000)])
def test_many_sequences_of_wide_tables_are_split(kv, heads, batch):
    """One of them may be long, and no group may read it alone."""
    scales = None if kv == N.BF16 else 1 << 20
    have = dict(kv=kv, R=512, batch=batch, heads=heads, scales=scales)
    for pages in (65, 2048, 8200):
        assert _attn(**have, stride=pages, ws=None, ws_bytes=0) == N.INVALID_ARG
        assert b"workspace too small" in N.load().last_error()
        rows = 16 if heads == 16 else heads  # of a unit, in whole row tiles
        assert _ws(kv, batch, 1, heads, 512, pages) >= (256 + batch) * rows * (512 + 2) * 4


@pytest.mark.parametrize("heads,seqs,rows,keys", [(20, 100, 6400, 12400), (16, 400, 25600, 50600),
                                                  (64, 60, 1920, 61920), (32, 5, 2000, 20000 + 2000),
                                                  (64, 33, 1000, 100000)])
def test_contexts_that_one_prompt_may_have_alone_are_split(heads, seqs, rows, keys):
    wide = dict(qs=heads * 192, ks=heads * 256, vs=heads * 256)
    assert _prompt(rows=rows, keys=keys, seqs=seqs, heads=heads, **wide, ws=None,
                   ws_bytes=0) == N.INVALID_ARG
    assert b"workspace too small" in N.load().last_error()
