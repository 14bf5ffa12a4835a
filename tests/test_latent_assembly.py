"""The attention over latents and of prompts, looked at in the assembly: nothing is spilled (a
reload in their loops would wait, as loads return in order, for the tile on its way), and LDS reads
are done, and loads into LDS counted, where a barrier hands a stage on."""

import os
import re
import subprocess

import pytest

from paper_2609_36899_amd import build
from test_lds_ring import _blocks, reads_at_barriers

SOURCES = ["attention_latent.hip", "attention_latent_few.hip", "attention_prompt.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """Kernel name -> (instruction lines, what the compiler says of it)."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path_factory.mktemp("asm")
    procs = [subprocess.Popen([build.HIPCC, *build.HIP_FLAGS, "-x", "hip", "--cuda-device-only", "-S",
                               os.path.join(build.CSRC, s), "-o", str(out / s)],
                              stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
             for s in SOURCES]
    assert [p.wait() for p in procs] == [0] * len(SOURCES)
    return {m[1]: (m[2], m[3]) for s in SOURCES for m in
            re.finditer(r"^(\w+):\s*; @\1\n(.*?)^\.Lfunc_end(.*?); COMPUTE_PGM_RSRC2:USER_SGPR",
                        (out / s).read_text(), re.M | re.S)}


@pytest.mark.parametrize("kernel,forms", [("latent_attn_kernel", 12), ("latent_few_kernel", 4),
                                          ("prompt_attn_kernel", 2), ("latent_merge_kernel", 3),
                                          ("prompt_merge_kernel", 2)])
def test_nothing_is_spilled(assembly, kernel, forms):
    found = {n: v for n, v in assembly.items() if kernel in n}
    assert len(found) >= forms
    for name, (body, facts) in found.items():
        assert re.search(r"; ScratchSize: 0\b", facts), name
        assert not re.search(r"^\s*(scratch_|buffer_(load|store)\S* .*off, s\[0:3\])", body, re.M), name


# Ahead of a piece the wide form may have reads of the sums of the one before in flight, which are no
# part of the ring: LDS takes what waves ask of it in order.
@pytest.mark.parametrize("kernel,forms,sums", [("latent_attn_kernel", 12, 1), ("latent_few_kernel", 4, 0),
                                               ("prompt_attn_kernel", 2, 0)])
def test_no_lds_read_in_flight_at_a_barrier(assembly, kernel, forms, sums):
    found = {n: v for n, v in assembly.items() if kernel in n}
    assert len(found) >= forms
    for name, (body, _) in found.items():
        left = sorted(reads_at_barriers(body))
        assert len(left) > sums and not any(left[:len(left) - sums]), (name, left)
