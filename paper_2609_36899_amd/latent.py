"""Binding of the operators over caller-owned pages of latents, of the attention of
prompts over what latents expand to, and of page copies (argument checks and
marshalling only; the calls are described in include/pdec.h).

As in paged.py, every tensor of a call lies on one GPU, the call goes to that GPU's
current stream unless one is given, and a workspace that is not given is allocated on
the call's stream.
"""

from __future__ import annotations

import ctypes
import functools
from typing import Optional, Sequence, Union

import torch

from . import _native as N
from ._native import PAGE_TOKENS
from .paged import (_BF16, _F32, _I32, _bad_tensor, _check, _dims, _handle, _ptr, _refuse, _run,
                    _workspace)

ROPE_DIM = 64  # of the rotary key that all heads share


def _pages(pages, scales):
    """(n_pages, latent width, kv dtype, device) of a pool of latents."""
    n, page, width = _dims(pages, "pages", 3)
    if pages.dtype is _BF16:
        kv, latent = N.BF16, width - ROPE_DIM
    elif pages.dtype is torch.uint8:
        kv, latent = N.FP8_E4M3, width - 2 * ROPE_DIM
    else:
        _refuse("pages must be bfloat16 or uint8 (E4M3 codes)")
    if n < 1 or page != PAGE_TOKENS or latent < 1:
        _refuse(f"pages hold {PAGE_TOKENS} tokens, each a latent and a rotary key")
    if not pages.is_contiguous():
        _refuse("pages must be contiguous")
    dev = pages.get_device()
    if kv == N.FP8_E4M3 and scales is not None:
        _check(scales, "scales", _F32, (n, PAGE_TOKENS), dev)
    elif kv == N.FP8_E4M3 or scales is not None:
        _refuse("E4M3 pages take scales, the others none")
    return n, latent, kv, dev


def _heads(t, name: str, dtype, shape, dev: int):
    """Row and head distance of rows of heads whose elements lie side by side."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _bad_tensor(t, name, dtype, shape, dev)
    n, h, d = shape
    row, head, one = t.stride()
    if h <= 1:
        head = d
    if n <= 1:
        row = max((h - 1) * head + d, d)
        row = (row + 7) // 8 * 8
    if n and h and (one != 1 or head < d or row < (h - 1) * head + d):
        _refuse(f"{name}'s elements must lie side by side, its heads and rows apart")
    return row, head


def _sequences(lens, row_start, block_table, dev: int):
    B = _dims(lens, "lens", 1)[0]
    _check(lens, "lens", _I32, (B,), dev)
    _check(row_start, "row_start", _I32, (B + 1,), dev)
    stride = _dims(block_table, "block_table", 2)[1]
    _check(block_table, "block_table", _I32, (B, stride), dev)
    return B, stride


def paged_latent_append(x: torch.Tensor, lens: torch.Tensor, row_start: torch.Tensor,
                        block_table: torch.Tensor, rope: torch.Tensor, pages: torch.Tensor,
                        scales: Optional[torch.Tensor] = None,
                        gain: Optional[torch.Tensor] = None, eps: float = 1e-6,
                        interleaved: bool = True, q: Optional[torch.Tensor] = None,
                        q_out: Optional[torch.Tensor] = None,
                        stream: Optional[torch.cuda.Stream] = None) -> None:
    """Norm, rotate and append the rows of x [rows][R + 64] (latent and rotary key, bf16
    or fp32, rows any distance apart) to caller-owned pages, and rotate q [rows][H][64]
    into q_out (bf16; heads and rows of both any distance apart, q_out may be q).

    lens int32 [B] counts the new tokens; row_start int32 [B + 1] says which rows are
    whose; block_table int32 [B][stride]; rope from rope_table(max_pos, 64).  Pages
    bfloat16 [P][16][R + 64], or uint8 [P][16][R + 128] with scales float32 [P][16];
    gain float32 [R], or None for no norm.
    """
    n_pages, latent, kv, dev = _pages(pages, scales)
    rows = _dims(x, "x", 2)[0]
    src = N.BF16 if x.dtype is _BF16 else N.F32
    dtype = _BF16 if src == N.BF16 else _F32
    shape = (rows, latent + ROPE_DIM)
    if x.dtype is not dtype or x.shape != shape or x.get_device() != dev:
        _bad_tensor(x, "x", dtype, shape, dev)
    x_stride, one = x.stride()
    if rows <= 1:
        x_stride = shape[1]
    if rows and (one != 1 or x_stride < shape[1]):
        _refuse("x's elements must lie side by side, its rows apart")
    B, stride = _sequences(lens, row_start, block_table, dev)
    max_pos = _dims(rope, "rope", 3)[0]
    _check(rope, "rope", _F32, (max_pos, ROPE_DIM // 2, 2), dev)
    if gain is not None:
        _check(gain, "gain", _F32, (latent,), dev)
    heads = q_row = q_head = out_row = out_head = 0
    if q is not None:
        heads = _dims(q, "q", 3)[1]
        q_row, q_head = _heads(q, "q", dtype, (rows, heads, ROPE_DIM), dev)
        _dims(q_out, "q_out", 3)
        out_row, out_head = _heads(q_out, "q_out", _BF16, (rows, heads, ROPE_DIM), dev)
    elif q_out is not None:
        _refuse("q and q_out come together")
    handle = _handle(dev, stream)
    if rows == 0:
        return
    _run(dev, N.load().paged_latent_append, src, kv, rows, B, heads, latent, x.data_ptr(),
         x_stride, _ptr(gain), float(eps), int(bool(interleaved)), _ptr(q), q_row, q_head,
         lens.data_ptr(), row_start.data_ptr(), block_table.data_ptr(), stride, n_pages,
         rope.data_ptr(), max_pos, _ptr(q_out), out_row, out_head, pages.data_ptr(),
         _ptr(scales), handle)


@functools.lru_cache(maxsize=1024)
def paged_latent_attention_workspace_bytes(kv_dtype: int, batch: int, n_q: int, n_heads: int,
                                           latent_dim: int, max_pages: int) -> int:
    """Scratch bytes for a table of max_pages pages, and for smaller batches, n_q and tables;
    kv_dtype BF16 or FP8_E4M3."""
    return N.check(N.load().paged_latent_attention_workspace_bytes(
        kv_dtype, batch, n_q, n_heads, latent_dim, max_pages))


def paged_latent_attention(q: torch.Tensor, pages: torch.Tensor, block_table: torch.Tensor,
                           lens: torch.Tensor, out: torch.Tensor, softmax_scale: float,
                           scales: Optional[torch.Tensor] = None,
                           workspace: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Attention of the last tokens of each sequence over caller-owned latents.

    q bfloat16 [B][n_q][H][R + 64] and out [B][n_q][H][R], or [B][H][..] for one token
    each; lens int32 [B] on the GPU, counting these tokens; pages bfloat16 [P][16][R +
    64], or uint8 [P][16][R + 128] with scales float32 [P][16]; softmax_scale that of
    the heads before they were absorbed.
    """
    n_pages, latent, kv, dev = _pages(pages, scales)
    four = isinstance(q, torch.Tensor) and q.dim() == 4
    shape = _dims(q, "q", 4 if four else 3)
    B, n_q, heads = shape[0], shape[1] if four else 1, shape[-2]
    _check(q, "q", _BF16, (*shape[:-1], latent + ROPE_DIM), dev)
    _check(out, "out", _BF16, (*shape[:-1], latent), dev)
    stride = _dims(block_table, "block_table", 2)[1]
    _check(block_table, "block_table", _I32, (B, stride), dev)
    _check(lens, "lens", _I32, (B,), dev)
    handle = _handle(dev, stream)
    ws, at, size = _workspace(
        workspace, paged_latent_attention_workspace_bytes(kv, B, n_q, heads, latent, stride), dev,
        stream)
    _run(dev, N.load().paged_latent_attention, kv, B, n_q, heads, latent, q.data_ptr(),
         pages.data_ptr(), _ptr(scales), n_pages, block_table.data_ptr(), stride,
         lens.data_ptr(), float(softmax_scale), out.data_ptr(), at, size, handle)
    return out


def paged_latent_rows(pages: torch.Tensor, lens: torch.Tensor, row_start: torch.Tensor,
                      block_table: torch.Tensor, latents: torch.Tensor, rope_keys: torch.Tensor,
                      scales: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """Cached tokens as rows: latents bfloat16 [rows][R] and rope_keys bfloat16 [rows][64].
    row_start int32 [B + 1] says which rows are whose, the last tokens of each sequence
    (with counts equal to lens, all of them)."""
    n_pages, latent, kv, dev = _pages(pages, scales)
    rows = _dims(latents, "latents", 2)[0]
    _check(latents, "latents", _BF16, (rows, latent), dev)
    _check(rope_keys, "rope_keys", _BF16, (rows, ROPE_DIM), dev)
    B, stride = _sequences(lens, row_start, block_table, dev)
    handle = _handle(dev, stream)
    if rows == 0:
        return
    _run(dev, N.load().paged_latent_rows, kv, rows, B, latent, pages.data_ptr(), _ptr(scales),
         lens.data_ptr(), row_start.data_ptr(), block_table.data_ptr(), stride, n_pages,
         latents.data_ptr(), rope_keys.data_ptr(), handle)


@functools.lru_cache(maxsize=1024)
def latent_prompt_attention_workspace_bytes(n_rows: int, n_seqs: int, n_heads: int,
                                            head_dim: int) -> int:
    """Scratch bytes for so many rows and sequences, and for fewer."""
    return N.check(N.load().latent_prompt_attention_workspace_bytes(n_rows, n_seqs, n_heads,
                                                                    head_dim))


def latent_prompt_attention(q: torch.Tensor, k: torch.Tensor, rope_keys: torch.Tensor,
                            v: torch.Tensor, q_start: torch.Tensor, k_start: torch.Tensor,
                            out: torch.Tensor, softmax_scale: float,
                            workspace: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Causal attention of prompts over expanded keys and values.

    q bfloat16 [rows][H][D + 64], k and v bfloat16 [keys][H][D] (heads and rows any
    distance apart: the halves of one projection's [keys][H][2 D] serve as they are),
    rope_keys bfloat16 [keys][64]; q_start and k_start int32 [B + 1]: whose rows and keys
    are whose, the last keys of a sequence its rows' own; out bfloat16 [rows][H][D].
    """
    rows, heads, dim = _dims(out, "out", 3)
    dev = out.get_device()
    _check(out, "out", _BF16, (rows, heads, dim), dev)
    _dims(q, "q", 3)
    q_row, q_head = _heads(q, "q", _BF16, (rows, heads, dim + ROPE_DIM), dev)
    keys = _dims(k, "k", 3)[0]
    k_row, k_head = _heads(k, "k", _BF16, (keys, heads, dim), dev)
    _dims(v, "v", 3)
    v_row, v_head = _heads(v, "v", _BF16, (keys, heads, dim), dev)
    _dims(rope_keys, "rope_keys", 2)
    if (rope_keys.dtype is not _BF16 or rope_keys.shape != (keys, ROPE_DIM)
            or rope_keys.get_device() != dev):
        _bad_tensor(rope_keys, "rope_keys", _BF16, (keys, ROPE_DIM), dev)
    r_row, one = rope_keys.stride()
    if keys <= 1:
        r_row = ROPE_DIM
    if keys and (one != 1 or r_row < ROPE_DIM):
        _refuse("rope_keys' elements must lie side by side, its rows apart")
    B = _dims(q_start, "q_start", 1)[0] - 1
    _check(q_start, "q_start", _I32, (B + 1,), dev)
    _check(k_start, "k_start", _I32, (B + 1,), dev)
    handle = _handle(dev, stream)
    ws, at, size = _workspace(
        workspace, latent_prompt_attention_workspace_bytes(rows, B, heads, dim), dev, stream)
    if rows == 0:
        return out
    _run(dev, N.load().latent_prompt_attention, rows, keys, B, heads, dim, q.data_ptr(), q_row,
         q_head, k.data_ptr(), k_row, k_head, rope_keys.data_ptr(), r_row, v.data_ptr(), v_row,
         v_head, q_start.data_ptr(), k_start.data_ptr(), float(softmax_scale), out.data_ptr(),
         at, size, handle)
    return out


def paged_copy_pages(pools: Union[torch.Tensor, Sequence[torch.Tensor]], src: torch.Tensor,
                     dst: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Copy entry src[i] of every pool (contiguous tensors [P][..] of any type: pages,
    scales, means) to its entry dst[i]; src and dst int32 [n] on the GPU.  No entry may be
    the destination of two pairs, or of one and the source of another."""
    if isinstance(pools, torch.Tensor):
        pools = [pools]
    n = _dims(src, "src", 1)[0]
    dev = src.get_device()
    _check(src, "src", _I32, (n,), dev)
    _check(dst, "dst", _I32, (n,), dev)
    if not pools:
        _refuse("no pools")
    places, sizes, n_pages = [], [], None
    for t in pools:
        if not isinstance(t, torch.Tensor) or t.dim() < 1 or t.get_device() != dev \
                or not t.is_contiguous():
            _refuse("pools must be contiguous tensors on the pairs' GPU")
        here, size = len(t), t.nbytes
        if n_pages is None:
            n_pages = here
        if here != n_pages or size == 0:
            _refuse("pools must have the same number of pages, and pages with something in them")
        places.append(t.data_ptr())
        sizes.append(size // n_pages)
    count = len(places)
    places = (ctypes.c_void_p * count)(*places)
    sizes = (ctypes.c_int64 * count)(*sizes)
    handle = _handle(dev, stream)
    if n == 0:
        return
    _run(dev, N.load().paged_copy_pages, count, places, sizes, n_pages, n, src.data_ptr(),
         dst.data_ptr(), handle)
