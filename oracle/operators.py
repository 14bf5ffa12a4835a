"""Operators over caller-owned pages and draft verification (oracle side).

TEST INFRASTRUCTURE ONLY (see the package docstring).

Plain float64 renderings of the definitions in include/pdec.h, a sequence and a
token at a time: appending rotated keys and values to pages, attention of the last
tokens of a sequence, the choice of pages, and the verification of drafted tokens.
Pages are in the library's layout, K [P][Hkv][16][Dh] and V [P][Hkv][Dh][16].
"""

from __future__ import annotations

import numpy as np

from .fp8 import e4m3_decode, e4m3_encode
from .sampling import token_masses

PAGE = 16


def rotate(x: np.ndarray, cs: np.ndarray) -> np.ndarray:
    """x [heads][Dh] turned by cs [Dh/2][2] = (cos, sin), pairs (i, i + Dh/2)."""
    half = x.shape[-1] // 2
    a, b = x[:, :half], x[:, half:]
    c, s = cs[:, 0], cs[:, 1]
    return np.concatenate([a * c - b * s, a * s + b * c], axis=1)


def page_scale(amax: float) -> float:
    """The smallest power of two, 2^-100 to 2^100, that brings amax to 448."""
    if not amax > 0:
        return 2.0 ** -100
    e = -100
    while e < 100 and amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def append_rows(k, v, lens, row_start, table, cs, limit, k_pages, v_pages, k_scales=None,
                v_scales=None, round_page=lambda x: x, q=None):
    """What paged_kv_append leaves: k_pages, v_pages (codes where scales are given), the
    scales, {(page, head): key mean}, and {row: rotated q}.  round_page rounds a value to
    the page type."""
    kp, vp = k_pages.copy(), v_pages.copy()
    ks = None if k_scales is None else k_scales.astype(np.float64)
    vs = None if v_scales is None else v_scales.astype(np.float64)
    means, q_rows = {}, {}
    for b in range(len(lens)):
        n = int(row_start[b + 1] - row_start[b])
        p = int(lens[b]) - n
        r = int(row_start[b])
        while r < row_start[b + 1]:
            slot = p % PAGE
            m = min(PAGE - slot, int(row_start[b + 1]) - r, limit - p)
            if p < 0:
                r, p = r + 1, p + 1
                continue
            if p >= limit:
                break
            if q is not None:
                for i in range(m):
                    q_rows[r + i] = rotate(q[r + i], cs[p + i])
            page = int(table[b][p // PAGE])
            if 0 <= page < kp.shape[0]:
                new_k = np.stack([rotate(k[r + i], cs[p + i]) for i in range(m)], axis=1)
                new_v = v[r:r + m].transpose(1, 2, 0)  # [head][dim][token]
                for g in range(kp.shape[1]):
                    if ks is None:
                        kp[page, g, slot:slot + m] = new_k[g]
                        vp[page, g, :, slot:slot + m] = new_v[g]
                        held = round_page(kp[page, g, :slot + m])
                    else:
                        for pages, scales, new, at in (
                                (kp, ks, new_k[g], np.s_[page, g, :slot]),
                                (vp, vs, new_v[g], np.s_[page, g, :, :slot])):
                            s = page_scale(float(np.abs(new).max()))
                            if slot > 0:
                                old = scales[page, g]
                                s = max(s, old)
                                if s != old:
                                    pages[at] = e4m3_encode(e4m3_decode(pages[at]) * old / s)
                            scales[page, g] = s
                        kp[page, g, slot:slot + m] = e4m3_encode(new_k[g] / ks[page, g])
                        vp[page, g, :, slot:slot + m] = e4m3_encode(new_v[g] / vs[page, g])
                        held = e4m3_decode(kp[page, g, :slot + m]) * ks[page, g]
                    means[page, g] = held.mean(axis=0)
            r, p = r + m, p + m
    return kp, vp, ks, vs, means, q_rows


def mix(q, k, v):
    """softmax(q k^T / sqrt(Dh)) v of one row q [Dh], and the same mix of |v|."""
    if len(k) == 0:
        return np.zeros(v.shape[1]), np.zeros(v.shape[1])
    s = k @ q / np.sqrt(len(q))
    w = np.exp(s - s.max())
    w /= w.sum()
    return w @ v, w @ np.abs(v)


def token_attention(q, k_pages, v_pages, table, lens, selected=None):
    """q [B][n_q][Hq][Dh] over pages of values (decoded): (out, mix of |v|)."""
    B, n_q, hq, dh = q.shape
    n_pages, hkv = k_pages.shape[:2]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    stride = table.shape[1]
    for b in range(B):
        n = min(max(int(lens[b]), 0), stride * PAGE)
        for g in range(hkv):
            if selected is None:
                pages = list(range(-(-n // PAGE)))
            else:
                pages = [int(p) for p in selected[b, g][:-(-n // PAGE)]]
            k, v, pos = [np.zeros((0, dh))], [np.zeros((0, dh))], [np.zeros(0, int)]
            for p in pages:
                if not 0 <= p < stride or not 0 <= table[b, p] < n_pages:
                    continue
                m = min(PAGE, n - p * PAGE)
                if m > 0:
                    k.append(k_pages[table[b, p], g, :m].astype(np.float64))
                    v.append(v_pages[table[b, p], g, :, :m].T.astype(np.float64))
                    pos.append(p * PAGE + np.arange(m))
            k, v, pos = np.concatenate(k), np.concatenate(v), np.concatenate(pos)
            for j in range(n_q):
                see = pos <= n - n_q + j
                for h in range(g * (hq // hkv), (g + 1) * (hq // hkv)):
                    out[b, j, h], size[b, j, h] = mix(q[b, j, h].astype(np.float64), k[see], v[see])
    return out, size


def select_pages(q, k_means, table, lens, n_selected, keep_first=1, keep_last=1):
    """Logical pages [B][Hkv][n_selected], ascending, -1 behind them."""
    B, hq, dh = q.shape
    n_pages, hkv = k_means.shape[:2]
    out = np.full((B, hkv, n_selected), -1, dtype=np.int32)
    big = np.finfo(np.float32).max
    for b in range(B):
        n = min(-(-max(int(lens[b]), 0) // PAGE), table.shape[1])
        for g in range(hkv):
            score = np.full(n, -float(big))
            for p in range(n):
                if 0 <= table[b, p] < n_pages:
                    s = q[b, g * (hq // hkv):(g + 1) * (hq // hkv)].astype(np.float64) @ \
                        k_means[table[b, p], g].astype(np.float64)
                    s = s[~np.isnan(s)]
                    if len(s):
                        score[p] = np.clip(np.float32(s.max()), -big, big)
            score[:keep_first] = np.inf
            score[max(n - keep_last, 0):] = np.inf
            best = np.argsort(-score, kind="stable")[:n_selected]
            out[b, g, :len(best)] = np.sort(best)
    return out


def _mass(z, temperature):
    z = np.asarray(z, dtype=np.float32).copy()
    z[np.isnan(z)] = -np.inf
    if not np.isfinite(z.max()):
        return np.zeros(z.shape, dtype=np.uint64), 0.0
    m = token_masses(z, temperature)
    return m, 2.0 ** 50 / float(int(m.sum(dtype=np.uint64)))


def _u24(u) -> int:
    u = np.float32(min(max(float(np.float32(u)), 0.0), float(np.nextafter(np.float32(1), np.float32(0)))))
    return int(np.floor(u * np.float32(2.0 ** 24)))


def verify_drafts(target, drafter, drafts, uniforms, temperature):
    """tokens [B][T + 1] (accepted drafts, the next token, then -1) and counts [B]."""
    B, T = drafts.shape
    V = target.shape[2]
    tokens, counts = np.full((B, T + 1), -1, dtype=np.int32), np.zeros(B, dtype=np.int32)
    for b in range(B):
        n, off = 0, None
        while True:
            mass, unit = _mass(target[b, n], temperature)
            p = mass.astype(np.float64) * unit
            if n == T or not 0 <= drafts[b, n] < V:
                break
            x = int(drafts[b, n])
            if drafter is None:
                d = np.zeros(V)
                d[x] = 2.0 ** 50
            else:
                mass, unit = _mass(drafter[b, n], temperature)
                d = mass.astype(np.float64) * unit
            if not float(_u24(uniforms[b, n])) * d[x] < 2.0 ** 24 * p[x]:
                off = d
                if drafter is None:
                    off[x] = np.inf
                break
            tokens[b, n] = x
            n += 1
        whole = np.rint(p).astype(np.int64)
        rest = whole if off is None else np.rint(np.maximum(p - off, 0.0)).astype(np.int64)
        if rest.sum() == 0:
            rest = whole
        z = int(rest.sum())
        goal = (_u24(uniforms[b, T]) * z) >> 24
        tokens[b, n] = int(np.argmax(np.cumsum(rest) > goal)) if z else 0
        counts[b] = n
    return tokens, counts
