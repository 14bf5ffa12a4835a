"""Binding of the operators over caller-owned pages and of draft verification
(argument checks and marshalling only; the calls are described in include/pdec.h).

Every tensor of a call lies on one GPU; without a stream the call goes to that
GPU's current one, whichever GPU is current.  A workspace that is not given is
allocated on the call's stream.  Wrong arguments raise PdecError before anything
is enqueued.
"""

from __future__ import annotations

import contextlib
from typing import Optional

import torch

from . import _native as N
from ._native import PAGE_TOKENS, PdecError

_KV_DTYPE = {torch.float32: N.F32, torch.bfloat16: N.BF16, torch.uint8: N.FP8_E4M3}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise PdecError(N.INVALID_ARG, what)


def _tensor(t, name: str, dtype, shape, device) -> None:
    """A contiguous GPU tensor of this type and shape (None: any size)."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda, f"{name} must be a GPU tensor")
    _need(device is None or t.device == device, f"{name} is on another device")
    _need(t.dtype == dtype, f"{name} must be {dtype}")
    _need(t.dim() == len(shape) and all(n is None or n == m for n, m in zip(shape, t.shape)),
          f"{name} must have shape {tuple('*' if n is None else n for n in shape)}, "
          f"not {tuple(t.shape)}")
    _need(t.is_contiguous(), f"{name} must be contiguous")


def _rows(t, name: str, heads, head_dim, device):
    """Rows of [heads][head_dim], any distance apart: what a slice of q|k|v rows is."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3,
          f"{name} must be a GPU tensor [rows][heads][head_dim]")
    _need(device is None or t.device == device, f"{name} is on another device")
    n, h, d = t.shape
    _need((heads is None or h == heads) and (head_dim is None or d == head_dim),
          f"{name} has other heads")
    _need(n == 0 or (t.stride(2) == 1 and (h == 1 or t.stride(1) == d)
                     and (n == 1 or t.stride(0) >= h * d)),
          f"{name}'s heads must lie side by side")
    return t.stride(0) if n > 1 else h * d


class _Call:
    """The device and stream of a call, and its workspace."""

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream]):
        self.device, self.stream = device, stream
        _need(stream is None or stream.device == device, "stream is on another device")
        self.guard = (contextlib.nullcontext() if torch.cuda.current_device() == device.index
                      else torch.cuda.device(device))
        s = stream if stream is not None else torch.cuda.current_stream(device)
        self.handle = s.cuda_stream

    def workspace(self, given: Optional[torch.Tensor], need: int) -> torch.Tensor:
        if given is not None:
            _need(given.is_cuda and given.device == self.device and given.is_contiguous(),
                  "workspace must be a contiguous tensor on the call's device")
            _need(given.numel() * given.element_size() >= need,
                  f"workspace too small: need {need} bytes")
            return given
        if self.stream is None:
            return torch.empty(need, dtype=torch.uint8, device=self.device)
        with torch.cuda.stream(self.stream):
            return torch.empty(need, dtype=torch.uint8, device=self.device)


def _pages(k_pages, v_pages, k_scales, v_scales, device):
    """(n_pages, n_kv_heads, head_dim, kv dtype) of a pool."""
    _need(isinstance(k_pages, torch.Tensor) and k_pages.dim() == 4, "k_pages must have 4 dims")
    n, hkv, page, dh = k_pages.shape
    _need(k_pages.dtype in _KV_DTYPE, "pages must be float32, bfloat16 or uint8 (E4M3 codes)")
    _need(n >= 1 and page == PAGE_TOKENS, f"pages hold {PAGE_TOKENS} tokens")
    _tensor(k_pages, "k_pages", k_pages.dtype, (n, hkv, PAGE_TOKENS, dh), device)
    _tensor(v_pages, "v_pages", k_pages.dtype, (n, hkv, dh, PAGE_TOKENS), k_pages.device)
    fp8 = k_pages.dtype == torch.uint8
    for t, name in ((k_scales, "k_scales"), (v_scales, "v_scales")):
        _need((t is not None) == fp8, "E4M3 pages take k_scales and v_scales, the others none")
        if fp8:
            _tensor(t, name, torch.float32, (n, hkv), k_pages.device)
    return n, hkv, dh, _KV_DTYPE[k_pages.dtype]


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def rope_table(max_pos: int, head_dim: int, base: float = 10000.0, device="cuda",
               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The (cos, sin) table [max_pos][head_dim / 2][2] that paged_kv_append rotates by."""
    _need(max_pos >= 1 and head_dim >= 2 and head_dim % 2 == 0, "bad rotary table size")
    device = torch.device(device)
    if device.index is None:
        device = torch.device("cuda", torch.cuda.current_device())
    call = _Call(device, stream)
    with call.guard, (torch.cuda.stream(stream) if stream is not None
                      else contextlib.nullcontext()):
        table = torch.empty((max_pos, head_dim // 2, 2), dtype=torch.float32, device=device)
        N.check(N.load().rope_table(max_pos, head_dim, float(base), table.data_ptr(),
                                    call.handle))
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
    n_pages, hkv, dh, kv = _pages(k_pages, v_pages, k_scales, v_scales, None)
    dev = k_pages.device
    k_stride = _rows(k, "k", hkv, dh, dev)
    v_stride = _rows(v, "v", hkv, dh, dev)
    rows = k.shape[0]
    _need(v.shape[0] == rows and k.dtype == v.dtype, "k and v must agree")
    _need(k.dtype in (torch.float32, torch.bfloat16), "rows must be float32 or bfloat16")
    _tensor(lens, "lens", torch.int32, (None,), dev)
    B = lens.shape[0]
    _tensor(row_start, "row_start", torch.int32, (B + 1,), dev)
    _tensor(block_table, "block_table", torch.int32, (B, None), dev)
    _tensor(rope, "rope", torch.float32, (None, dh // 2, 2), dev)
    _need((q is None) == (q_out is None), "q and q_out come together")
    hq, q_stride = 0, 0
    if q is not None:
        q_stride = _rows(q, "q", None, dh, dev)
        hq = q.shape[1]
        _need(q.shape[0] == rows and q.dtype == k.dtype, "q and k must agree")
        _tensor(q_out, "q_out", torch.float32 if kv == N.F32 else torch.bfloat16, (rows, hq, dh),
                dev)
    if k_means is not None:
        _tensor(k_means, "k_means", torch.bfloat16, (n_pages, hkv, dh), dev)
    call = _Call(dev, stream)
    if rows == 0:
        return
    with call.guard:
        N.check(N.load().paged_kv_append(
            N.F32 if k.dtype == torch.float32 else N.BF16, kv, rows, B, hq, hkv, dh, _ptr(q),
            q_stride, k.data_ptr(), k_stride, v.data_ptr(), v_stride, lens.data_ptr(),
            row_start.data_ptr(), block_table.data_ptr(), block_table.shape[1], n_pages,
            rope.data_ptr(), rope.shape[0], _ptr(q_out), k_pages.data_ptr(), v_pages.data_ptr(),
            _ptr(k_scales), _ptr(v_scales), _ptr(k_means), call.handle))


def paged_token_attention_workspace_bytes(batch: int, n_q: int, n_q_heads: int, n_kv_heads: int,
                                          head_dim: int) -> int:
    return N.check(N.load().paged_token_attention_workspace_bytes(batch, n_q, n_q_heads,
                                                                  n_kv_heads, head_dim))


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
    n_pages, hkv, dh, kv = _pages(k_pages, v_pages, k_scales, v_scales, None)
    dev = k_pages.device
    _need(kv != N.F32, "pages must be bfloat16 or uint8")
    _need(isinstance(q, torch.Tensor) and q.dim() in (3, 4), "q must be [B][n_q][Hq][Dh]")
    B, hq, n_q = q.shape[0], q.shape[-2], q.shape[1] if q.dim() == 4 else 1
    _tensor(q, "q", torch.bfloat16, (*q.shape[:-1], dh), dev)
    _tensor(out, "out", torch.bfloat16, tuple(q.shape), dev)
    _tensor(block_table, "block_table", torch.int32, (B, None), dev)
    _tensor(lens, "lens", torch.int32, (B,), dev)
    if selected is not None:
        _need(n_q == 1, "selected pages take one query token")
        _tensor(selected, "selected", torch.int32, (B, hkv, None), dev)
    lib = N.load()
    call = _Call(dev, stream)
    with call.guard:
        ws = call.workspace(workspace, N.check(
            lib.paged_token_attention_workspace_bytes(B, n_q, hq, hkv, dh)))
        N.check(lib.paged_token_attention(
            kv, B, n_q, hq, hkv, dh, q.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
            _ptr(k_scales), _ptr(v_scales), n_pages, block_table.data_ptr(),
            block_table.shape[1], lens.data_ptr(), _ptr(selected),
            0 if selected is None else selected.shape[2], out.data_ptr(), ws.data_ptr(),
            ws.numel() * ws.element_size(), call.handle))
    return out


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
    _need(isinstance(k_means, torch.Tensor) and k_means.dim() == 3, "k_means must have 3 dims")
    n_pages, hkv, dh = k_means.shape
    _tensor(k_means, "k_means", torch.bfloat16, (None, hkv, dh), None)
    dev = k_means.device
    _tensor(q, "q", torch.bfloat16, (None, None, dh), dev)
    B, hq, _ = q.shape
    _tensor(block_table, "block_table", torch.int32, (B, None), dev)
    _tensor(lens, "lens", torch.int32, (B,), dev)
    _tensor(selected, "selected", torch.int32, (B, hkv, None), dev)
    lib = N.load()
    call = _Call(dev, stream)
    stride = block_table.shape[1]
    with call.guard:
        ws = call.workspace(workspace, N.check(lib.paged_select_workspace_bytes(B, hkv, stride)))
        N.check(lib.paged_select(
            B, hq, hkv, dh, q.data_ptr(), k_means.data_ptr(), n_pages, block_table.data_ptr(),
            stride, lens.data_ptr(), selected.shape[2], int(keep_first), int(keep_last),
            selected.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), call.handle))
    return selected


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
    _tensor(target_logits, "target_logits", torch.float32, (None, None, None), None)
    dev = target_logits.device
    B, rows, V = target_logits.shape
    n = rows - 1
    _tensor(draft_tokens, "draft_tokens", torch.int32, (B, n), dev)
    _tensor(uniforms, "uniforms", torch.float32, (B, rows), dev)
    _tensor(tokens_out, "tokens_out", torch.int32, (B, rows), dev)
    _tensor(accepted_out, "accepted_out", torch.int32, (B,), dev)
    if draft_logits is not None:
        _tensor(draft_logits, "draft_logits", torch.float32, (B, n, V), dev)
    lib = N.load()
    call = _Call(dev, stream)
    with call.guard:
        ws = call.workspace(workspace, N.check(
            lib.verify_drafts_workspace_bytes(B, n, V, int(draft_logits is not None))))
        N.check(lib.verify_drafts(
            B, n, V, target_logits.data_ptr(), _ptr(draft_logits), draft_tokens.data_ptr(),
            uniforms.data_ptr(), float(temperature), tokens_out.data_ptr(),
            accepted_out.data_ptr(), ws.data_ptr(), ws.numel() * ws.element_size(), call.handle))
    return tokens_out
