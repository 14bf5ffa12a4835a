"""Latent operators over long caches and far addresses, and calls side by side.

A long table repeats the pages of a small pool, so that the float64 result follows from each
page's count; tolerances as in test_gpu_latent_attention.py."""

import numpy as np
import pytest
import torch

from oracle.fp8 import e4m3_decode
from test_gpu_latent_attention import Case
from test_gpu_latent_prompt import Prompt

pytestmark = pytest.mark.gpu
ROPE = 64


def _P():
    import paper_2609_36899_amd as P
    return P


@pytest.mark.parametrize("heads", [2, 20, 100])
@pytest.mark.parametrize("latent,fp8", [(256, True), (256, False), (512, True), (512, False)])
def test_stretches_of_many_pages(latent, fp8, heads):
    """More than a million keys: each group's piece is longer than the ids that it holds at once."""
    rng = np.random.default_rng(latent + heads)
    B, n_pages, pool = 3, 30000, 400
    table = rng.integers(0, pool, (B, n_pages)).astype(np.int32)
    lens = np.array([n_pages * 16, (n_pages - 4321) * 16, (n_pages - 7) * 16], np.int32)
    rope = torch.from_numpy(rng.standard_normal((pool, 16, ROPE)).astype(np.float32)).bfloat16()
    scales = None
    if fp8:
        codes = rng.integers(0, 127, (pool, 16, latent)).astype(np.uint8)
        codes |= (rng.integers(0, 2, codes.shape) << 7).astype(np.uint8)
        ts = np.exp2(rng.integers(-9, -5, (pool, 16))).astype(np.float32)
        c = e4m3_decode(codes).astype(np.float64) * ts[..., None]
        pages = torch.from_numpy(np.concatenate([codes, rope.view(torch.uint8).numpy()], -1)).cuda()
        scales = torch.from_numpy(ts).cuda()
    else:
        latents = torch.from_numpy(rng.standard_normal((pool, 16, latent)).astype(np.float32)).bfloat16()
        c = latents.double().numpy()
        pages = torch.cat([latents, rope], -1).cuda()
    q = torch.from_numpy(rng.standard_normal((B, heads, latent + ROPE)).astype(np.float32)).bfloat16()
    out = torch.empty((B, heads, latent), dtype=torch.bfloat16, device="cuda")
    scale = 0.07
    _P().paged_latent_attention(q.cuda(), pages, torch.from_numpy(table).cuda(),
                                torch.from_numpy(lens).cuda(), out, scale, scales=scales)
    keys = np.concatenate([c, rope.double().numpy()], -1).reshape(-1, latent + ROPE)
    c = c.reshape(-1, latent)
    for b in range(B):
        count = np.repeat(np.bincount(table[b, :lens[b] // 16], minlength=pool), 16)
        qb = q[b].double().numpy()
        s = scale * qb @ keys.T
        w = np.exp(s - s.max(-1, keepdims=True)) * count
        w /= w.sum(-1, keepdims=True)
        want, size = w @ c, w @ np.abs(c)
        reach = scale * (np.abs(qb) @ np.abs(keys).T).max(-1)
        E = 2.0 ** -24 * (latent + 68) * reach + 2.0 ** -22 + 2.0 ** -24 * (lens[b] + 64)
        both = size + np.abs(want)
        tol = 2.0 ** -8 * (both + np.abs(want)) + E[:, None] * both
        assert (np.abs(out[b].double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("heads", [3, 40])
@pytest.mark.parametrize("fp8", [False, True])
def test_pages_past_32_bits(fp8, heads):
    case = Case([700, 33], heads, 1, 512, fp8, seed=21)
    a = case.args()
    per = a["pages"][0].numel() * a["pages"].element_size()
    far = (1 << 32) // per + 5  # pages ahead of the case's
    big = torch.empty((far + case.P, *a["pages"].shape[1:]), dtype=a["pages"].dtype, device="cuda")
    big[far:] = a["pages"]
    a.update(pages=big, block_table=a["block_table"] + far)
    if fp8:
        scales = torch.full((far + case.P, 16), float("nan"), device="cuda")
        scales[far:] = a["scales"]
        a.update(scales=scales)
    case.check(_P().paged_latent_attention(**a))


def test_prompt_keys_past_32_bits():
    case = Prompt([90], [150], 1, 64, seed=22)
    a = case.args()
    wide = torch.empty((150, 1 << 24), dtype=torch.bfloat16, device="cuda")
    wide[:, :128] = case.kv.cuda()[:, 0]
    kv = wide[:, None, :128]
    a.update(k=kv[..., :64], v=kv[..., 64:])
    case.check(_P().latent_prompt_attention(**a))


@pytest.mark.parametrize("heads", [8, 64])
def test_calls_side_by_side(heads):
    """Two streams at once, each call with a workspace of its own."""
    P = _P()
    cases = [Case([5000, 300, 77], heads, 1, 256, fp8, seed=23 + fp8) for fp8 in (False, True)]
    prompts = [Prompt([300, 40], [700, 50], 4, 128, seed=25 + i) for i in range(2)]
    args = [(c.args(), p.args()) for c, p in zip(cases, prompts)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (a, p) in zip(streams, args):
            P.paged_latent_attention(**a, stream=s)
            P.latent_prompt_attention(**p, stream=s)
    torch.cuda.synchronize()
    for c, p, (a, b) in zip(cases, prompts, args):
        c.check(a["out"])
        p.check(b["out"])


def test_two_graphs_of_one_workspace():
    """Replayed in turn on one stream, with eager calls between them."""
    P = _P()
    cases = [Case([4000, 90], 16, 1, 256, False, seed=27), Case([900, 2600, 5], 40, 1, 256, True, seed=28)]
    args = [c.args() for c in cases]
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    stream, graphs = torch.cuda.Stream(), []
    stream.wait_stream(torch.cuda.current_stream())
    for a in args:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            P.paged_latent_attention(**a, workspace=ws)
    for _ in range(3):
        for c, a, g in zip(cases, args, graphs):
            a["out"].zero_()
            g.replay()
            got = a["out"].clone()
            c.check(got)
            assert torch.equal(got, c.run(workspace=ws))
