"""A workspace serves every smaller call: the sizes that the library asks for grow with each of
their arguments, across the sizes from which work is split in another way."""

import pytest

from paper_2609_36899_amd import _native as N

BATCHES = [1, 2, 64, 511, 512, 2047, 2048, 5000]


@pytest.mark.parametrize("kv", [N.BF16, N.FP8_E4M3])
@pytest.mark.parametrize("heads", [1, 5, 16, 17, 64, 128, 1024])
def test_latent_attention(kv, heads):
    fn = N.load().paged_latent_attention_workspace_bytes
    sizes = {(b, q, p): fn(kv, b, q, heads, 512, p)
             for b in BATCHES for q in (1, 2, 3, 7, 8, 26, 128) for p in (1, 7, 8, 16, 17, 1000)}
    assert min(sizes.values()) >= 0
    for (b, q, p), have in sizes.items():
        for (b1, q1, p1), need in sizes.items():
            if b1 <= b and q1 <= q and p1 <= p:
                assert need <= have, (b, q, p, b1, q1, p1)


@pytest.mark.parametrize("heads", [1, 20, 300, 512, 1024])
def test_latent_prompts(heads):
    fn = N.load().latent_prompt_attention_workspace_bytes
    sizes = {(r, s): fn(r, s, heads, 128) for r in (0, 1, 128, 4096, 1 << 20) for s in (1, 5, 1000)}
    assert min(sizes.values()) >= 0
    for (r, s), have in sizes.items():
        for (r1, s1), need in sizes.items():
            if r1 <= r and s1 <= s:
                assert need <= have, (r, s, r1, s1)
