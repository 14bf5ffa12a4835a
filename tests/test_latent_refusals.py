"""What the calls over pages of latents and paged_copy_pages refuse, on the host: no launch
is made, so made-up addresses serve as pointers."""

import ctypes

import pytest
import torch

from paper_2609_36899_amd import _native as N
from paper_2609_36899_amd import latent
from paper_2609_36899_amd._native import PdecError

A = 1 << 20  # a made-up, aligned address


def _append(**kw):
    a = dict(src=N.BF16, kv=N.BF16, rows=4, seqs=2, heads=4, R=256, x=A, xs=320, gain=A, eps=1e-6,
             inter=1, q=A, qs=256, qh=64, lens=A, start=A, bt=A, stride=8, pages=9, rope=A,
             max_pos=50, qo=A, qos=256, qoh=64, pool=A, scales=None)
    a.update(kw)
    return N.load().paged_latent_append(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(src=2), N.INVALID_ARG, b"src_dtype"), (dict(kv=N.F32), N.INVALID_ARG, b"kv_dtype"),
    (dict(R=384), N.UNSUPPORTED, b"latent_dim"), (dict(R=0), N.UNSUPPORTED, b"latent_dim"),
    (dict(x=None), N.INVALID_ARG, b"null"), (dict(pool=None), N.INVALID_ARG, b"null"),
    (dict(qo=None), N.INVALID_ARG, b"null"), (dict(q=None), N.INVALID_ARG, b"null"),
    (dict(lens=None), N.INVALID_ARG, b"null"), (dict(seqs=0), N.INVALID_ARG, b"batch"),
    (dict(stride=0), N.INVALID_ARG, b"bt_stride"), (dict(pages=1 << 31), N.INVALID_ARG, b"n_pages"),
    (dict(rows=-1), N.INVALID_ARG, b"n_rows"), (dict(max_pos=0), N.INVALID_ARG, b"max_pos"),
    (dict(inter=2), N.INVALID_ARG, b"interleaved"), (dict(eps=-1.0), N.INVALID_ARG, b"eps"),
    (dict(eps=float("nan")), N.INVALID_ARG, b"eps"), (dict(xs=319), N.INVALID_ARG, b"strides"),
    (dict(qs=255), N.INVALID_ARG, b"strides"), (dict(qh=63), N.INVALID_ARG, b"strides"),
    (dict(qos=255), N.INVALID_ARG, b"strides"), (dict(heads=0), N.INVALID_ARG, b"n_heads"),
    (dict(scales=A), N.INVALID_ARG, b"scales"), (dict(kv=N.FP8_E4M3), N.INVALID_ARG, b"scales"),
    (dict(pool=A + 8), N.INVALID_ARG, b"aligned"), (dict(gain=A + 4), N.INVALID_ARG, b"aligned"),
    (dict(rows=1 << 30), N.INVALID_ARG, b"too many rows"),
])
def test_append(kw, code, word):
    assert _append(**kw) == code
    assert word in N.load().last_error()


def test_no_rows_are_nothing():
    assert _append(rows=0) == N.OK and _rows(rows=0) == N.OK and _prompt(rows=0) == N.OK
    assert _copy(pairs=0, src=None) == N.OK


def _rows(**kw):
    a = dict(kv=N.BF16, rows=4, seqs=2, R=256, pool=A, scales=None, lens=A, start=A, bt=A, stride=8,
             pages=9, c=A, k=A)
    a.update(kw)
    return N.load().paged_latent_rows(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(kv=0), N.INVALID_ARG, b"kv_dtype"), (dict(R=128), N.UNSUPPORTED, b"latent_dim"),
    (dict(k=None), N.INVALID_ARG, b"null"), (dict(rows=-1), N.INVALID_ARG, b"n_rows"),
    (dict(c=A + 2), N.INVALID_ARG, b"aligned"), (dict(kv=2), N.INVALID_ARG, b"scales"),
    (dict(seqs=-1), N.INVALID_ARG, b"batch"),
])
def test_rows(kw, code, word):
    assert _rows(**kw) == code
    assert word in N.load().last_error()


def _attn(**kw):
    a = dict(kv=N.BF16, batch=2, n_q=1, heads=4, R=256, q=A, pool=A, scales=None, pages=9, bt=A,
             stride=800, lens=A, scale=0.1, out=A, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return N.load().paged_latent_attention(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(kv=0), N.INVALID_ARG, b"kv_dtype"), (dict(R=320), N.UNSUPPORTED, b"latent_dim"),
    (dict(q=None), N.INVALID_ARG, b"null"), (dict(ws=None), N.INVALID_ARG, b"too small"),
    (dict(n_q=0), N.INVALID_ARG, b"n_q"), (dict(n_q=4097), N.INVALID_ARG, b"n_q"),
    (dict(heads=0), N.INVALID_ARG, b"n_heads"), (dict(heads=1025), N.INVALID_ARG, b"n_heads"),
    (dict(batch=0), N.INVALID_ARG, b"batch"), (dict(scales=A), N.INVALID_ARG, b"scales"),
    (dict(kv=2), N.INVALID_ARG, b"scales"), (dict(scale=0.0), N.INVALID_ARG, b"softmax_scale"),
    (dict(scale=float("inf")), N.INVALID_ARG, b"softmax_scale"),
    (dict(out=A + 2), N.INVALID_ARG, b"aligned"), (dict(ws_bytes=100), N.INVALID_ARG, b"too small"),
    (dict(batch=1 << 20, stride=1 << 22), N.INVALID_ARG, b"too large"),
    (dict(batch=1 << 14, n_q=4096, heads=1024, stride=1), N.INVALID_ARG, b"too large"),
])
def test_attention(kw, code, word):
    assert _attn(**kw) == code
    assert word in N.load().last_error()


def _prompt(**kw):
    a = dict(rows=4, keys=9, seqs=2, heads=4, dim=128, q=A, qs=768, qh=192, k=A, ks=1024, kh=256,
             r=A, rs=64, v=A, vs=1024, vh=256, q0=A, k0=A, scale=0.1, out=A, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return N.load().latent_prompt_attention(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(dim=96), N.UNSUPPORTED, b"head_dim"), (dict(rows=-1), N.INVALID_ARG, b"n_rows"),
    (dict(keys=-1), N.INVALID_ARG, b"n_keys"), (dict(seqs=0), N.INVALID_ARG, b"n_seqs"),
    (dict(heads=0), N.INVALID_ARG, b"n_heads"), (dict(q=None), N.INVALID_ARG, b"null"),
    (dict(v=None), N.INVALID_ARG, b"null"), (dict(k0=None), N.INVALID_ARG, b"null"),
    (dict(scale=-1.0), N.INVALID_ARG, b"softmax_scale"), (dict(qs=767), N.INVALID_ARG, b"strides"),
    (dict(kh=127), N.INVALID_ARG, b"strides"), (dict(vs=890), N.INVALID_ARG, b"strides"),
    (dict(rs=63), N.INVALID_ARG, b"strides"), (dict(ks=1028), N.INVALID_ARG, b"aligned"),
    (dict(q=A + 2), N.INVALID_ARG, b"aligned"), (dict(rs=(1 << 24) + 8), N.INVALID_ARG, b"2^24"),
    (dict(ws_bytes=100), N.INVALID_ARG, b"too small"), (dict(ws=None), N.INVALID_ARG, b"too small"),
    (dict(rows=(1 << 31) - 1, keys=(1 << 31) - 1), N.INVALID_ARG, b"too many"),
])
def test_prompt(kw, code, word):
    assert _prompt(**kw) == code
    assert word in N.load().last_error()


def _copy(n_pools=2, pools=(A, A), sizes=(64, 32), pages=9, pairs=3, src=A, dst=A):
    count = max(len(pools), 1)
    return N.load().paged_copy_pages(n_pools, (ctypes.c_void_p * count)(*pools),
                                     (ctypes.c_int64 * count)(*sizes), pages, pairs, src, dst, None)


@pytest.mark.parametrize("kw,word", [
    (dict(n_pools=0), b"n_pools"), (dict(pages=0), b"n_pages"), (dict(pairs=-1), b"n_pairs"),
    (dict(src=None), b"null"), (dict(pools=(A, None)), b"null"), (dict(sizes=(64, 0)), b"bytes"),
    (dict(sizes=((1 << 27) + 1, 4)), b"bytes"), (dict(pairs=1 << 25), b"too many pairs"),
    (dict(pools=(A + 1, A), sizes=(1 << 27, 4)), b"unaligned"),
])
def test_copy(kw, word):
    assert _copy(**kw) == N.INVALID_ARG
    assert word in N.load().last_error()


def _ws(kv=N.BF16, batch=2, n_q=1, heads=4, R=256, max_pages=800):
    return N.load().paged_latent_attention_workspace_bytes(kv, batch, n_q, heads, R, max_pages)


def test_workspaces_serve_smaller_sizes():
    """What fewer sequences, tokens or pages take is never more."""
    for kv in (N.BF16, N.FP8_E4M3):
        for R in (256, 512):
            for heads in (1, 5, 16, 33, 64, 100, 128, 200):
                last = 0
                for batch in (1, 2, 17, 100, 255, 256, 400, 511, 512, 600, 5000):
                    now = _ws(kv, batch, 1, heads, R)
                    assert now >= last
                    last = now
                for batch in (1, 200, 600):
                    sizes = [_ws(kv, batch, n_q, heads, R) for n_q in range(1, 40)]
                    assert sizes == sorted(sizes)
                    sizes = [_ws(kv, batch, 2, heads, R, p) for p in (1, 8, 9, 16, 17, 100, 4000)]
                    assert sizes == sorted(sizes)
    fn = N.load().latent_prompt_attention_workspace_bytes
    for heads in (1, 7, 128, 1000):
        sizes = [fn(n, s, heads, 128) for n, s in ((0, 1), (9, 1), (5000, 1), (5000, 900), (90000, 900))]
        assert sizes == sorted(sizes)
    for bad in (dict(kv=0), dict(R=100), dict(batch=0), dict(n_q=5000), dict(heads=0), dict(max_pages=0)):
        assert _ws(**bad) < 0
    assert fn(-1, 1, 1, 128) < 0 and fn(1, 0, 1, 128) < 0 and fn(1, 1, 1, 100) < 0


def test_binding_refuses_what_is_no_gpu_tensor():
    x = torch.zeros(4, 320, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int32)
    pool = torch.zeros(2, 16, 320, dtype=torch.bfloat16)
    with pytest.raises(PdecError, match="pages"):
        latent.paged_latent_append(x, i, i, i, x, pool)
    with pytest.raises(PdecError, match="pages"):
        latent.paged_latent_attention(x, pool, i, i, x, 0.1)
    with pytest.raises(PdecError, match="pages"):
        latent.paged_latent_rows(pool, i, i, i, x, x)
    with pytest.raises(PdecError, match="out"):
        latent.latent_prompt_attention(x, x, x, x, i, i, x, 0.1)
    with pytest.raises(PdecError, match="src"):
        latent.paged_copy_pages(pool, i, i)
    with pytest.raises(PdecError, match="src"):
        latent.paged_copy_pages(pool, None, i)
