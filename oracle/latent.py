"""Operators over pages of latents (oracle side).

TEST INFRASTRUCTURE ONLY (see the package docstring).

Plain float64 renderings of the definitions in include/pdec.h, a row or a sequence at
a time: latents normed and rotary keys rotated into pages, attention in the absorbed
and the expanded form, and page copies.  A pool is held as values: latents
[P][16][R], rotary keys [P][16][64], and scales [P][16] where the latents are codes.
"""

from __future__ import annotations

import numpy as np

from .operators import page_scale

PAGE, ROPE = 16, 64


def norm(x, gain, eps):
    """x over the root of its mean square, times gain (None: x)."""
    if gain is None:
        return x
    return x / np.sqrt(np.mean(x * x) + eps) * gain


def rotate(x, cs, interleaved):
    """x [..][64] turned by cs [32][2] = (cos, sin)."""
    c, s = cs[:, 0], cs[:, 1]
    out = np.empty_like(x)
    a, b = (np.s_[..., 0::2], np.s_[..., 1::2]) if interleaved else (np.s_[..., :32], np.s_[..., 32:])
    out[a] = x[a] * c - x[b] * s
    out[b] = x[a] * s + x[b] * c
    return out


def rows(lens, row_start, table, limit, n_pages, n_rows):
    """(row, sequence, position, page or None) of each row that has a position."""
    for b in range(len(lens)):
        for r in range(max(int(row_start[b]), 0), min(int(row_start[b + 1]), n_rows)):
            pos = int(lens[b]) - (int(row_start[b + 1]) - r)
            if 0 <= pos < limit:
                page = int(table[b, pos // PAGE])
                yield r, b, pos, page if 0 <= page < n_pages else None


def append(x, lens, row_start, table, cs, limit, n_pages, gain, eps, interleaved, scaled, q=None):
    """({(page, slot): (latent, rotary key, scale or None)}, {row: rotated q}), latents over
    their scale where scaled."""
    R = x.shape[1] - ROPE
    slots, q_rows = {}, {}
    for r, b, pos, page in rows(lens, row_start, table, limit, n_pages, len(x)):
        if q is not None:
            q_rows[r] = rotate(q[r], cs[pos], interleaved)
        if page is None:
            continue
        c = norm(x[r, :R], gain, eps)
        scale = page_scale(np.max(np.abs(c))) if scaled else None
        slots[page, pos % PAGE] = (c / scale if scaled else c,
                                   rotate(x[r, R:], cs[pos], interleaved), scale)
    return slots, q_rows


def mix(q, k, v, scale, seen):
    """softmax(scale q k^T) v of rows q [n][D] over the keys that seen [n][L] says, and the
    same mix of |v|; rows that see nothing give zeros."""
    out, size = np.zeros((len(q), v.shape[1])), np.zeros((len(q), v.shape[1]))
    with np.errstate(invalid="ignore"):
        s = np.where(seen, (q @ k.T) * scale, -np.inf)
        for i in range(len(q)):
            at = np.flatnonzero(seen[i])
            if len(at):
                w = np.exp(s[i, at] - np.max(s[i, at]))
                w /= w.sum()
                out[i], size[i] = w @ v[at], w @ np.abs(v[at])
    return out, size


def attention(q, latents, keys, table, lens, scale):
    """q [B][n_q][H][R + 64] over latents [P][16][R] and keys [P][16][64] (values as they read
    back): the outputs, their sizes (the same mix of |c|), and max sum |q k| scale a row."""
    B, n_q, H, _ = q.shape
    R, n_pages = latents.shape[2], latents.shape[0]
    out, size = np.zeros((B, n_q, H, R)), np.zeros((B, n_q, H, R))
    reach = np.zeros((B, n_q, H))
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * PAGE)
        pages = table[b, :-(-n // PAGE)]
        there = np.repeat((pages >= 0) & (pages < n_pages), PAGE)[:n]
        ids = np.where((pages >= 0) & (pages < n_pages), pages, 0)
        c = latents[ids].reshape(-1, R)[:n]
        k = np.concatenate([c, keys[ids].reshape(-1, ROPE)[:n]], axis=1)
        for j in range(n_q):
            m = n - n_q + j + 1
            if m <= 0:
                continue
            seen = np.broadcast_to(there & (np.arange(n) < m), (H, n))
            out[b, j], size[b, j] = mix(q[b, j], k, c, scale, seen)
            if seen[0].any():
                at = np.flatnonzero(seen[0])
                reach[b, j] = np.max(np.abs(q[b, j]) @ np.abs(k[at]).T, axis=1) * scale
    return out, size, reach


def prompt(q, k, rope_keys, v, q_start, k_start, scale):
    """The expanded form: q [T][H][D + 64], k and v [S][H][D]; outputs, sizes and reach as
    attention's, [T][H][..]."""
    T, H, D = q.shape[0], q.shape[1], k.shape[2]
    out, size, reach = np.zeros((T, H, D)), np.zeros((T, H, D)), np.zeros((T, H))
    for b in range(len(q_start) - 1):
        r, s = np.s_[q_start[b]:q_start[b + 1]], np.s_[k_start[b]:k_start[b + 1]]
        nq, nk = q_start[b + 1] - q_start[b], k_start[b + 1] - k_start[b]
        seen = np.arange(nk)[None] <= (nk - nq + np.arange(nq))[:, None]
        for h in range(H):
            keys = np.concatenate([k[s, h], rope_keys[s]], axis=1)
            out[r, h], size[r, h] = mix(q[r, h], keys, v[s, h], scale, seen)
            if nk:
                top = np.where(seen, np.abs(q[r, h]) @ np.abs(keys).T, 0.0)
                reach[r, h] = np.max(top, axis=1, initial=0.0) * scale
    return out, size, reach
