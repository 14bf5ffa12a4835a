"""Binding of the operators over caller-owned pages and of draft verification
(argument checks and marshalling only; the calls are described in include/pdec.h).

Every tensor of a call lies on one GPU; without a stream the call goes to that
GPU's current one, whichever GPU is current.  A workspace that is not given is
allocated on the call's stream.  Wrong arguments raise PdecError before anything
is enqueued.
"""

from __future__ import annotations

import contextlib
import functools
from typing import Optional

import torch

from . import _native as N
from ._native import PAGE_TOKENS, PdecError

_KV_DTYPE = {torch.float32: N.F32, torch.bfloat16: N.BF16, torch.uint8: N.FP8_E4M3}
_F32, _BF16, _I32 = torch.float32, torch.bfloat16, torch.int32

# A decode step makes these calls many times a millisecond, so what is right is found by
# few, cheap looks at a tensor, and what is wrong with it only then.


def _refuse(what: str):
    raise PdecError(N.INVALID_ARG, what)


def _bad_tensor(t, name: str, dtype, shape, dev: int):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a GPU tensor")
    if t.get_device() != dev:
        _refuse(f"{name} is on another device")
    if t.dtype != dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        _refuse(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    _refuse(f"{name} must be contiguous")


def _check(t, name: str, dtype, shape, dev: int) -> None:
    """A contiguous tensor of this type and shape on GPU dev."""
    try:
        if (t.dtype is dtype and t.shape == shape and t.get_device() == dev
                and t.is_contiguous()):
            return
    except AttributeError:  # no tensor
        pass
    _bad_tensor(t, name, dtype, shape, dev)


def _dims(t, name: str, n: int):
    """The sizes of a GPU tensor of n dims."""
    try:
        if t.get_device() >= 0:
            shape = t.shape
            if len(shape) == n:
                return shape
    except AttributeError:  # no tensor
        pass
    _refuse(f"{name} must be a GPU tensor of {n} dims")


def _rows(t, name: str, dtype, shape, dev: int) -> int:
    """Row distance of rows of [heads][head_dim], any distance apart: what a slice of
    q|k|v rows is."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        _bad_tensor(t, name, dtype, shape, dev)
    n, h, d = shape
    row, head, one = t.stride()
    if not (one == 1 and (head == d or h == 1) and (row >= h * d or n <= 1)) and n:
        _refuse(f"{name}'s heads must lie side by side in a row")
    return row if n > 1 else h * d


def _handle(dev: int, stream: Optional[torch.cuda.Stream]) -> int:
    """The stream handle of a call on GPU dev."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        _refuse("stream is on another device")
    return stream.cuda_stream


def _workspace(given: Optional[torch.Tensor], need: int, dev: int,
               stream: Optional[torch.cuda.Stream]):
    """(tensor, address, bytes) of a call's workspace."""
    if given is None:
        if need == 0:
            return None, None, 0
        if stream is None:
            given = torch.empty(need, dtype=torch.uint8, device=dev)
        else:
            with torch.cuda.stream(stream):
                given = torch.empty(need, dtype=torch.uint8, device=dev)
        return given, given.data_ptr(), need
    if given.get_device() != dev or not given.is_contiguous():
        _refuse("workspace must be a contiguous tensor on the call's device")
    have = given.numel() * given.element_size()
    if have < need:
        _refuse(f"workspace too small: need {need} bytes")
    return given, given.data_ptr(), have


def _run(dev: int, fn, *args) -> None:
    if torch._C._cuda_getDevice() == dev:
        rc = fn(*args)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args)
    if rc < 0:
        N.check(rc)


def _pages(k_pages, v_pages, k_scales, v_scales):
    """(n_pages, n_kv_heads, head_dim, kv dtype, device) of a pool."""
    n, hkv, page, dh = _dims(k_pages, "k_pages", 4)
    kv = _KV_DTYPE.get(k_pages.dtype)
    if kv is None:
        _refuse("pages must be float32, bfloat16 or uint8 (E4M3 codes)")
    if n < 1 or page != PAGE_TOKENS:
        _refuse(f"pages hold {PAGE_TOKENS} tokens")
    dev = k_pages.get_device()
    if not k_pages.is_contiguous():
        _refuse("k_pages must be contiguous")
    _check(v_pages, "v_pages", k_pages.dtype, (n, hkv, dh, PAGE_TOKENS), dev)
    if kv == N.FP8_E4M3 and k_scales is not None and v_scales is not None:
        _check(k_scales, "k_scales", _F32, (n, hkv), dev)
        _check(v_scales, "v_scales", _F32, (n, hkv), dev)
    elif kv == N.FP8_E4M3 or k_scales is not None or v_scales is not None:
        _refuse("E4M3 pages take k_scales and v_scales, the others none")
    return n, hkv, dh, kv, dev


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def rope_table(max_pos: int, head_dim: int, base: float = 10000.0, device="cuda",
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The (cos, sin) table [max_pos][head_dim / 2][2] that paged_kv_append rotates by."""
    if not 1 <= max_pos < 1 << 31 or head_dim < 2 or head_dim % 2:
        _refuse("bad rotary table size")
    if torch.device(device).type != "cuda":
        _refuse("the rotary table is made on a GPU")
    index = torch.device(device).index
    dev = torch.cuda.current_device() if index is None else index
    handle = _handle(dev, stream)
    with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
        table = torch.empty((max_pos, head_dim // 2, 2), dtype=_F32, device=dev)
    _run(dev, N.load().rope_table, max_pos, head_dim, float(base), table.data_ptr(), handle)
    return table


def paged_kv_append(k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor,
                    row_start: torch.Tensor, block_table: torch.Tensor, rope: torch.Tensor,
                    k_pages: torch.Tensor, v_pages: torch.Tensor,
                    k_scales: Optional[torch.Tensor] = None,
                    v_scales: Optional[torch.Tensor] = None,
                    k_means: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
                    q_out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> None:
    """Rotate and append the rows of k and v [rows][Hkv][Dh] (bf16 or fp32, slices of
    wider rows too) to caller-owned pages, and rotate q [rows][Hq][Dh] into q_out.

    lens int32 [B] counts the new tokens; row_start int32 [B + 1] says which rows are
    whose; block_table int32 [B][stride]; rope from rope_table.  Pages float32, bfloat16
    or uint8 (E4M3 codes, with k_scales and v_scales float32 [P][Hkv], which the call
    keeps); k_means bfloat16 [P][Hkv][Dh], kept where given.
    """
    n_pages, hkv, dh, kv, dev = _pages(k_pages, v_pages, k_scales, v_scales)
    rows = _dims(k, "k", 3)[0]
    src = N.BF16 if k.dtype is _BF16 else N.F32
    dtype = _BF16 if src == N.BF16 else _F32
    k_stride = _rows(k, "k", dtype, (rows, hkv, dh), dev)
    _dims(v, "v", 3)
    v_stride = _rows(v, "v", dtype, (rows, hkv, dh), dev)
    B = _dims(lens, "lens", 1)[0]
    _check(lens, "lens", _I32, (B,), dev)
    _check(row_start, "row_start", _I32, (B + 1,), dev)
    stride = _dims(block_table, "block_table", 2)[1]
    _check(block_table, "block_table", _I32, (B, stride), dev)
    max_pos = _dims(rope, "rope", 3)[0]
    _check(rope, "rope", _F32, (max_pos, dh // 2, 2), dev)
    hq = q_stride = 0
    if q is not None:
        hq = _dims(q, "q", 3)[1]
        q_stride = _rows(q, "q", dtype, (rows, hq, dh), dev)
        _check(q_out, "q_out", _F32 if kv == N.F32 else _BF16, (rows, hq, dh), dev)
    elif q_out is not None:
        _refuse("q and q_out come together")
    if k_means is not None:
        _check(k_means, "k_means", _BF16, (n_pages, hkv, dh), dev)
    handle = _handle(dev, stream)
    if rows == 0:
        return
    _run(dev, N.load().paged_kv_append, src, kv, rows, B, hq, hkv, dh, _ptr(q), q_stride,
             k.data_ptr(), k_stride, v.data_ptr(), v_stride, lens.data_ptr(),
             row_start.data_ptr(), block_table.data_ptr(), stride, n_pages, rope.data_ptr(),
             max_pos, _ptr(q_out), k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales),
             _ptr(v_scales), _ptr(k_means), handle)


@functools.lru_cache(maxsize=1024)
def paged_token_attention_workspace_bytes(batch: int, n_q: int, n_q_heads: int, n_kv_heads: int,
                                          head_dim: int, max_pages: int) -> int:
    """Scratch bytes for a table (or a selection, if that is smaller) of max_pages pages, and
    for smaller batches, n_q and tables."""
    return N.check(N.load().paged_token_attention_workspace_bytes(
        batch, n_q, n_q_heads, n_kv_heads, head_dim, max_pages))


def paged_token_attention(q: torch.Tensor, k_pages: torch.Tensor, v_pages: torch.Tensor,
                          block_table: torch.Tensor, lens: torch.Tensor, out: torch.Tensor,
                          k_scales: Optional[torch.Tensor] = None,
                          v_scales: Optional[torch.Tensor] = None,
                          selected: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Attention of the last tokens of each sequence over caller-owned pages.

    q and out bfloat16 [B][n_q][Hq][Dh], or [B][Hq][Dh] for one token each; lens int32
    [B] on the GPU, counting these tokens; pages bfloat16, or uint8 (E4M3 codes) with
    k_scales and v_scales float32 [P][Hkv]; selected int32 [B][Hkv][n], one token each:
    the logical pages to read instead of all.
    """
    n_pages, hkv, dh, kv, dev = _pages(k_pages, v_pages, k_scales, v_scales)
    if kv == N.F32:
        _refuse("pages must be bfloat16 or uint8")
    four = isinstance(q, torch.Tensor) and q.dim() == 4
    shape = _dims(q, "q", 4 if four else 3)
    B, n_q, hq = shape[0], shape[1] if four else 1, shape[-2]
    want = (*shape[:-1], dh)
    _check(q, "q", _BF16, want, dev)
    _check(out, "out", _BF16, want, dev)
    stride = _dims(block_table, "block_table", 2)[1]
    _check(block_table, "block_table", _I32, (B, stride), dev)
    _check(lens, "lens", _I32, (B,), dev)
    n_sel = 0
    if selected is not None:
        if n_q != 1:
            _refuse("selected pages take one query token")
        n_sel = _dims(selected, "selected", 3)[2]
        _check(selected, "selected", _I32, (B, hkv, n_sel), dev)
    handle = _handle(dev, stream)
    ws, at, size = _workspace(
        workspace, paged_token_attention_workspace_bytes(
            B, n_q, hq, hkv, dh, stride if selected is None else min(stride, n_sel)), dev, stream)
    _run(dev, N.load().paged_token_attention, kv, B, n_q, hq, hkv, dh, q.data_ptr(),
             k_pages.data_ptr(), v_pages.data_ptr(), _ptr(k_scales), _ptr(v_scales), n_pages,
             block_table.data_ptr(), stride, lens.data_ptr(), _ptr(selected), n_sel,
             out.data_ptr(), at, size, handle)
    return out


@functools.lru_cache(maxsize=1024)
def paged_select_workspace_bytes(batch: int, n_kv_heads: int, bt_stride: int) -> int:
    return N.check(N.load().paged_select_workspace_bytes(batch, n_kv_heads, bt_stride))


def paged_select(q: torch.Tensor, k_means: torch.Tensor, block_table: torch.Tensor,
                 lens: torch.Tensor, selected: torch.Tensor, keep_first: int = 1,
                 keep_last: int = 1, workspace: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The pages of largest score q . mean of each sequence and KV head, into selected
    int32 [B][Hkv][n], in page order (see paged_select in include/pdec.h).

    q bfloat16 [B][Hq][Dh], k_means bfloat16 [P][Hkv][Dh] as paged_kv_append keeps
    them, block_table int32 [B][stride] and lens int32 [B] on the GPU."""
    n_pages, hkv, dh = _dims(k_means, "k_means", 3)
    dev = k_means.get_device()
    _check(k_means, "k_means", _BF16, (n_pages, hkv, dh), dev)
    B, hq, _ = _dims(q, "q", 3)
    _check(q, "q", _BF16, (B, hq, dh), dev)
    stride = _dims(block_table, "block_table", 2)[1]
    _check(block_table, "block_table", _I32, (B, stride), dev)
    _check(lens, "lens", _I32, (B,), dev)
    n_sel = _dims(selected, "selected", 3)[2]
    _check(selected, "selected", _I32, (B, hkv, n_sel), dev)
    if not (0 <= keep_first <= n_sel and 1 <= keep_last <= n_sel):
        _refuse("keep_first >= 0, keep_last >= 1 and their sum at most n_selected")
    handle = _handle(dev, stream)
    ws, at, size = _workspace(workspace, paged_select_workspace_bytes(B, hkv, stride), dev, stream)
    _run(dev, N.load().paged_select, B, hq, hkv, dh, q.data_ptr(), k_means.data_ptr(), n_pages,
             block_table.data_ptr(), stride, lens.data_ptr(), n_sel, int(keep_first),
             int(keep_last), selected.data_ptr(), at, size, handle)
    return selected


@functools.lru_cache(maxsize=1024)
def verify_drafts_workspace_bytes(batch: int, n_drafts: int, vocab: int,
                                  with_drafter: bool) -> int:
    return N.check(N.load().verify_drafts_workspace_bytes(batch, n_drafts, vocab,
                                                          int(bool(with_drafter))))


def verify_drafts(target_logits: torch.Tensor, draft_tokens: torch.Tensor,
                  uniforms: torch.Tensor, tokens_out: torch.Tensor, accepted_out: torch.Tensor,
                  temperature: float = 1.0, draft_logits: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Accept or refuse drafted tokens and draw the next one (see verify_drafts in
    include/pdec.h).

    target_logits float32 [B][n + 1][V], draft_tokens int32 [B][n], uniforms float32
    [B][n + 1], draft_logits float32 [B][n][V] or None; tokens_out int32 [B][n + 1],
    accepted_out int32 [B]."""
    B, rows, V = _dims(target_logits, "target_logits", 3)
    n, dev = rows - 1, target_logits.get_device()
    _check(target_logits, "target_logits", _F32, (B, rows, V), dev)
    _check(draft_tokens, "draft_tokens", _I32, (B, n), dev)
    _check(uniforms, "uniforms", _F32, (B, rows), dev)
    _check(tokens_out, "tokens_out", _I32, (B, rows), dev)
    _check(accepted_out, "accepted_out", _I32, (B,), dev)
    if draft_logits is not None:
        _check(draft_logits, "draft_logits", _F32, (B, n, V), dev)
    handle = _handle(dev, stream)
    ws, at, size = _workspace(
        workspace, verify_drafts_workspace_bytes(B, n, V, draft_logits is not None), dev, stream)
    _run(dev, N.load().verify_drafts, B, n, V, target_logits.data_ptr(), _ptr(draft_logits),
             draft_tokens.data_ptr(), uniforms.data_ptr(), float(temperature),
             tokens_out.data_ptr(), accepted_out.data_ptr(), at, size, handle)
    return tokens_out
