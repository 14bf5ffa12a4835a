"""Operators of models whose cache is one latent vector a token, and what they are measured on.

Five kinds of case, each through the package's public entry points:

  append     paged_latent_append: new tokens' latents, normed, and rotary keys, rotated at
             their positions, into their page slots; the queries' rotary parts on the way
  attention  paged_latent_attention: one or several query tokens per trajectory over the
             latents themselves (the absorbed form)
  rows       paged_latent_rows: cached latents and rotary keys as rows, for the projection
             that expands them
  prompt     latent_prompt_attention: a prompt's tokens over expanded keys and values
  copy       paged_copy_pages: pages of a pool to other places in it

`run` computes them in plain torch operations, or, with `own`, through the package.

Pages hold 16 tokens. A token's row is its latent, then its rotary key of 64 elements: bf16
throughout, or the latent as E4M3 codes (one byte each) that read back as code * scale, a
power of two for each token, and the rotary key in bf16.
"""

import math

import numpy as np
import torch

own = False

PAGE = 16
ROPE = 64
DEV = "cuda"
F8 = torch.float8_e4m3fn
EPS = 1e-6


def listed():
    return [
        # One token for each trajectory of a decode batch, 8-bit pages, one of four shares of
        # the heads.
        dict(name="append_decode_e4m3_b64", kind="append", pages="e4m3", src="bf16", batch=64,
             heads=32, latent=512, interleaved=True, lo=1024, hi=8192, new_lo=1, new_hi=1,
             draw_seed=1),
        # A prompt in one pass, from a projection's fp32 output.
        dict(name="append_prompt_bf16_4096", kind="append", pages="bf16", src="f32", batch=1,
             heads=32, latent=512, interleaved=False, lo=0, hi=0, new_lo=4096, new_hi=4096,
             draw_seed=2),
        # The smallest decode call: a few short trajectories of a small model, latency alone.
        dict(name="attention_bf16_b4_short", kind="attention", pages="bf16", batch=4, heads=4,
             latent=256, nq=1, lo=1, hi=128, draw_seed=1),
        # A mid-sized decode batch, one of eight shares of the heads.
        dict(name="attention_e4m3_b64_h16", kind="attention", pages="e4m3", batch=64, heads=16,
             latent=512, nq=1, lo=1024, hi=8192, draw_seed=21),
        # The same batch with all heads on one card.
        dict(name="attention_bf16_b64_h128", kind="attention", pages="bf16", batch=64, heads=128,
             latent=512, nq=1, lo=1024, hi=8192, draw_seed=21),
        # Few very long contexts, each with its last token and three drafted ones.
        dict(name="attention_e4m3_b8_long_nq4", kind="attention", pages="e4m3", batch=8,
             heads=32, latent=512, nq=4, lo=65536, hi=131072, draw_seed=3),
        # One trajectory's cached tokens, an odd number of them.
        dict(name="rows_bf16_b1", kind="rows", pages="bf16", batch=1, latent=512, lo=2001,
             hi=2001, draw_seed=1),
        # What four tool outputs are appended to.
        dict(name="rows_e4m3_b4", kind="rows", pages="e4m3", batch=4, latent=512, lo=4096,
             hi=16384, draw_seed=4),
        # A prompt alone, one of several shares of the heads.
        dict(name="prompt_b1_4096_h20", kind="prompt", batch=1, heads=20, dim=128, lo=0, hi=0,
             new_lo=4096, new_hi=4096, draw_seed=1),
        # Tool outputs of five trajectories over what they hold already.
        dict(name="prompt_b5_turns_h32", kind="prompt", batch=5, heads=32, dim=128, lo=1000,
             hi=6000, new_lo=100, new_hi=700, draw_seed=2),
        # Group rollouts of a prompt: its part-full page for each of its forks.
        dict(name="copy_fork_b64", kind="copy", pages="e4m3", latent=512, pairs=64, sources=8,
             draw_seed=1),
        # Half of a fragmented pool moved together.
        dict(name="copy_compact_8k", kind="copy", pages="bf16", latent=512, pairs=8190,
             sources=8190, draw_seed=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "attention", "rows", "prompt",
                       "prompt", "copy"])
    seed = rng.randrange(1 << 20)
    latent = rng.choice([512, 512, 256])
    pages = rng.choice(["e4m3", "bf16"])
    heads = rng.choice([16, 16, 128, 128, 64, 32, 20, 8, 5, 1])
    if kind == "append":
        batch = _log_int(rng, 1, 128)
        new = _log_int(rng, 1, max(2, 4000 // batch)) if rng.random() < 0.6 else 1
        return dict(kind=kind, pages=pages, src=rng.choice(["bf16", "f32"]), batch=batch,
                    heads=rng.choice([1, 5, 8, 20, 32, 64]), latent=latent, interleaved=rng.random() < 0.5, lo=0,
                    hi=_log_int(rng, 16, 8192), new_lo=max(1, new // 4), new_hi=new,
                    draw_seed=seed)
    if kind == "attention":
        batch, nq = _log_int(rng, 1, 96), rng.choice([1, 1, 2, 3, 4, 7])
        most = min(500000, 90000000 // (heads * nq)) // batch
        hi = min(131072, _log_int(rng, 64, max(most, 128)))
        return dict(kind=kind, pages=pages, batch=batch, heads=heads, latent=latent, nq=nq,
                    lo=max(1, hi // rng.choice([1, 2, 8, 64])), hi=hi, draw_seed=seed)
    if kind == "rows":
        batch = _log_int(rng, 1, 64)
        hi = _log_int(rng, 16, 60000 // batch)
        return dict(kind=kind, pages=pages, batch=batch, latent=latent,
                    lo=max(1, hi // rng.choice([1, 4, 16])), hi=hi, draw_seed=seed)
    if kind == "prompt":
        batch = _log_int(rng, 1, 16)
        new = _log_int(rng, 1, 4000 // batch)
        heads = rng.choice([5, 8, 10, 20, 32])
        most = 200000000 // (heads * new * batch)  # keys that keep a pass below the longest
        return dict(kind=kind, batch=batch, heads=heads, dim=rng.choice([128, 128, 64]), lo=0,
                    hi=_log_int(rng, 16, max(16, min(16000 // batch, most - new))),
                    new_lo=max(1, new // 4), new_hi=new, draw_seed=seed)
    pairs = _log_int(rng, 1, 8000)
    return dict(kind=kind, pages=pages, latent=latent, pairs=pairs,
                sources=max(1, pairs // rng.choice([1, 1, 8])), draw_seed=seed)


# ---- sizes that follow from a case alone ------------------------------------

def _pages(n):
    return (n + PAGE - 1) // PAGE


def _lens(case):
    """Cached tokens of each trajectory, the new ones among them, and the new ones."""
    rng = np.random.default_rng(case["draw_seed"])
    ctx = rng.integers(case["lo"], case["hi"] + 1, size=case["batch"])
    if "new_lo" in case:
        new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["batch"])
        return ctx + new, new
    return ctx, None


def _row_bytes(case):
    """A cached token's bytes, its scale among them."""
    return (case["latent"] + ROPE) * 2 if case["pages"] == "bf16" else case["latent"] + 2 * ROPE + 4


def work(case):
    kind = case["kind"]
    if kind == "copy":
        by = (case["sources"] + case["pairs"]) * PAGE * _row_bytes(case)
        return {"bytes": by + case["pairs"] * 8, "flops": 0}
    lens, new = _lens(case)
    if kind == "append":
        n, heads, r = int(new.sum()), case["heads"], case["latent"]
        src = 2 if case["src"] == "bf16" else 4
        by = n * (r + ROPE) * src + n * _row_bytes(case)     # rows in, page slots out
        by += n * heads * ROPE * (src + 2)                   # rotary queries
        by += n * ROPE * 4 + r * 4                           # rotation table, gain
        return {"bytes": by, "flops": n * (4 * r + 3 * (heads + 1) * ROPE)}
    if kind == "rows":
        n = int(lens.sum())
        return {"bytes": n * (_row_bytes(case) + (case["latent"] + ROPE) * 2), "flops": 0}
    if kind == "attention":
        r, rows, keys = case["latent"], case["nq"] * case["heads"], int(lens.sum())
        by = keys * _row_bytes(case) + case["batch"] * rows * (2 * r + ROPE) * 2
        return {"bytes": by, "flops": 2 * keys * rows * (2 * r + ROPE)}
    heads, d = case["heads"], case["dim"]
    by = int(new.sum()) * heads * (2 * d + ROPE) * 2
    by += int(lens.sum()) * (heads * 2 * d + ROPE) * 2
    pairs = int((new * lens - new * (new - 1) // 2).sum())   # a token sees those up to itself
    return {"bytes": by, "flops": 2 * pairs * heads * (2 * d + ROPE)}


# ---- inputs ------------------------------------------------------------------

def _rope_table(max_pos):
    """(cos, sin) of each position and pair, angles in 64 bits."""
    inv = 10000.0 ** (-2.0 * torch.arange(ROPE // 2, dtype=torch.float64, device=DEV) / ROPE)
    ang = torch.arange(max_pos, dtype=torch.float64, device=DEV)[:, None] * inv
    return torch.stack([ang.cos(), ang.sin()], dim=-1).float().contiguous()


def _pool(case, g, pool):
    """Pages of `pool` places, full of tokens as an append leaves them, and their scales."""
    r = case["latent"]
    if case["pages"] == "bf16":
        return torch.randn((pool, PAGE, r + ROPE), dtype=torch.bfloat16, device=DEV,
                           generator=g), None
    pages = torch.empty((pool, PAGE, r + 2 * ROPE), dtype=torch.uint8, device=DEV)
    for a in range(0, pool, 4096):  # what is made on the way stays small
        part = pages[a:a + 4096]
        x = torch.randn((*part.shape[:2], r + ROPE), dtype=torch.bfloat16, device=DEV, generator=g)
        codes = (x[..., :r].float() * 100.0).clamp_(-448.0, 448.0)
        part[..., :r] = codes.to(F8).view(torch.uint8)
        part[..., r:] = x[..., r:].contiguous().view(torch.uint8)
    e = torch.randint(-8, -5, (pool, PAGE), device=DEV, generator=g)
    return pages, torch.exp2(e.float())


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "copy":
        n, m = case["pairs"], case["sources"]
        st = dict(case=case)
        st["pages"], st["scales"] = _pool(case, g, n + m + 3)
        perm = torch.randperm(n + m + 3, device=DEV, generator=g).int()
        st["src"] = perm[torch.arange(n, device=DEV) % m].contiguous()
        st["dst"] = perm[m:m + n].contiguous()
        return st
    lens, new = _lens(case)
    B = case["batch"]
    st = dict(case=case, host_lens=[int(x) for x in lens])
    if new is not None:
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        st["host_starts"] = [int(x) for x in starts]
        st["starts"] = torch.from_numpy(starts).to(DEV)
    if kind == "prompt":
        heads, d = case["heads"], case["dim"]
        n, total = int(new.sum()), int(lens.sum())
        ends = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        st["host_ends"] = [int(x) for x in ends]
        st["key_starts"] = torch.from_numpy(ends).to(DEV)
        st["q"] = torch.randn((n, heads, d + ROPE), dtype=torch.bfloat16, device=DEV, generator=g)
        # Keys and values side by side for each head, as one projection of the latents leaves them.
        st["kv"] = torch.randn((total, heads, 2 * d), dtype=torch.bfloat16, device=DEV, generator=g)
        st["rope_keys"] = torch.randn((total, ROPE), dtype=torch.bfloat16, device=DEV, generator=g)
        st["out"] = torch.empty((n, heads, d), dtype=torch.bfloat16, device=DEV)
        return st

    r = case["latent"]
    n_pages = _pages(lens)
    pool = int(n_pages.sum()) + 3
    perm = torch.randperm(pool, device=DEV, generator=g).int()
    stride = int(n_pages.max()) + 1
    at = np.concatenate([[0], np.cumsum(n_pages)[:-1]])[:, None] + np.arange(stride)[None]
    used = np.arange(stride)[None] < n_pages[:, None]
    at = torch.from_numpy(np.where(used, at, 0)).to(DEV)
    st["table"] = torch.where(torch.from_numpy(used).to(DEV), perm[at],
                              torch.zeros_like(perm[:1])).contiguous()
    st["lens"] = torch.from_numpy(lens.astype(np.int32)).to(DEV)
    st["pages"], st["scales"] = _pool(case, g, pool)
    if kind == "append":
        n, heads = int(new.sum()), case["heads"]
        td = torch.bfloat16 if case["src"] == "bf16" else torch.float32
        st["rope"] = _rope_table(int(lens.max()))
        # Rows of differing size: the norm evens them out.
        size = torch.exp2(torch.randn((n, 1), device=DEV, generator=g))
        st["x"] = torch.randn((n, r + ROPE), device=DEV, generator=g).mul_(size).to(td)
        st["gain"] = 1.0 + 0.2 * torch.randn(r, device=DEV, generator=g)
        # The rotary part is the end of each head of the query projection's rows, and goes
        # behind the absorbed part of the query that the attention takes.
        st["heads"] = torch.randn((n, heads, 128 + ROPE), dtype=td, device=DEV, generator=g)
        st["q"] = torch.randn((n, heads, r + ROPE), dtype=torch.bfloat16, device=DEV, generator=g)
        return st
    if kind == "rows":
        n = int(lens.sum())
        starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        st["host_starts"] = [int(x) for x in starts]
        st["starts"] = torch.from_numpy(starts).to(DEV)
        st["latents"] = torch.empty((n, r), dtype=torch.bfloat16, device=DEV)
        st["rope_keys"] = torch.empty((n, ROPE), dtype=torch.bfloat16, device=DEV)
        return st
    shape = (B, case["nq"], case["heads"])
    st["q"] = torch.randn((*shape, r + ROPE), dtype=torch.bfloat16, device=DEV, generator=g)
    st["out"] = torch.empty((*shape, r), dtype=torch.bfloat16, device=DEV)
    st["softmax_scale"] = (128 + ROPE) ** -0.5  # of the heads before they were absorbed
    return st


# ---- one pass ------------------------------------------------------------------

def run(state):
    return {"append": _append, "attention": _attention, "rows": _rows, "prompt": _prompt,
            "copy": _copy}[state["case"]["kind"]](state)


def _parts(st):
    """Views of the pool's pages: latents (as codes of E4M3 pages) and rotary keys."""
    r, pages = st["case"]["latent"], st["pages"]
    if st["scales"] is None:
        return pages[..., :r], pages[..., r:]
    return pages[..., :r].view(F8), pages[..., r:].view(torch.bfloat16)


def _append(st):
    case, r = st["case"], st["case"]["latent"]
    q_in, q_out = st["heads"][..., 128:], st["q"][..., r:]
    if own:
        import paper_2609_36899_amd as P
        P.paged_latent_append(st["x"], st["lens"], st["starts"], st["table"], st["rope"],
                              st["pages"], scales=st["scales"], gain=st["gain"], eps=EPS,
                              interleaved=case["interleaved"], q=q_in, q_out=q_out)
    else:
        _append_plain(st, q_in, q_out)
    latents, keys = _parts(st)
    return {"q": q_out, "latents": latents, "rope_keys": keys, "scales": st["scales"]}


def _rotate(x, cs, interleaved):
    x = x.float()
    c, s = cs[..., 0], cs[..., 1]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * c - b * s, a * s + b * c], dim=-1).flatten(-2)
    a, b = x[..., :ROPE // 2], x[..., ROPE // 2:]
    return torch.cat([a * c - b * s, a * s + b * c], dim=-1)


def _append_plain(st, q_in, q_out):
    case, r = st["case"], st["case"]["latent"]
    starts, lens = st["starts"].long(), st["lens"].long()
    row = torch.arange(st["x"].shape[0], device=DEV)
    seq = torch.searchsorted(starts[1:], row, right=True)
    pos = lens[seq] - (starts[seq + 1] - row)
    page, slot = st["table"][seq, pos // PAGE].long(), pos % PAGE
    cs = st["rope"][pos]
    q_out.copy_(_rotate(q_in, cs[:, None], case["interleaved"]))
    x = st["x"][:, :r].float()
    c = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * st["gain"]
    k = _rotate(st["x"][:, r:], cs, case["interleaved"]).to(torch.bfloat16)
    latents, keys = _parts(st)
    if st["scales"] is None:
        latents[page, slot] = c.to(torch.bfloat16)
    else:
        m, e = torch.frexp(c.abs().amax(-1))  # the least power of two that brings it to 448
        e = e - 9 + (m > 0.875).int()
        e = torch.where(m > 0, e, torch.full_like(e, -100)).clamp(-100, 100)
        scale = torch.ldexp(torch.ones_like(m), e)
        codes = (c / scale[:, None]).clamp(-448, 448).to(F8).view(torch.uint8)
        st["pages"][..., :r][page, slot] = codes
        st["scales"][page, slot] = scale
    keys[page, slot] = k


def _softmax_mix(s, v):
    """softmax(s) v over the last axis of s, rows of -inf throughout giving zeros."""
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m.masked_fill(m == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v) / total.masked_fill(total == 0, 1.0)


def _attention(st):
    if own:
        import paper_2609_36899_amd as P
        return P.paged_latent_attention(st["q"], st["pages"], st["table"], st["lens"], st["out"],
                                        st["softmax_scale"], scales=st["scales"])
    B, nq, heads, width = st["q"].shape
    ids = st["table"].long()
    latents, keys = _parts(st)
    if st["scales"] is None:
        c = latents[ids].float()
    else:
        c = latents.view(torch.uint8)[ids].view(F8).float() * st["scales"][ids][..., None]
    c = c.reshape(B, -1, width - ROPE)
    k = torch.cat([c, keys[ids].float().reshape(B, -1, ROPE)], dim=-1)
    pos = torch.arange(k.shape[1], device=DEV)
    last = st["lens"].long()[:, None] - nq + torch.arange(nq, device=DEV)[None, :]
    seen = (pos[None, None, :] <= last[:, :, None]).repeat_interleave(heads, dim=1)
    s = torch.matmul(st["q"].float().reshape(B, nq * heads, width), k.transpose(1, 2))
    s = (s * st["softmax_scale"]).masked_fill(~seen, -math.inf)
    st["out"].copy_(_softmax_mix(s, c).reshape(st["out"].shape))
    return st["out"]


def _rows(st):
    if own:
        import paper_2609_36899_amd as P
        P.paged_latent_rows(st["pages"], st["lens"], st["starts"], st["table"], st["latents"],
                            st["rope_keys"], scales=st["scales"])
        return st["latents"], st["rope_keys"]
    starts, lens = st["starts"].long(), st["lens"].long()
    row = torch.arange(st["latents"].shape[0], device=DEV)
    seq = torch.searchsorted(starts[1:], row, right=True)
    pos = lens[seq] - (starts[seq + 1] - row)
    page, slot = st["table"][seq, pos // PAGE].long(), pos % PAGE
    latents, keys = _parts(st)
    if st["scales"] is None:
        st["latents"].copy_(latents[page, slot])
    else:
        codes = latents.view(torch.uint8)[page, slot].view(F8)
        st["latents"].copy_(codes.float() * st["scales"][page, slot][:, None])
    st["rope_keys"].copy_(keys[page, slot])
    return st["latents"], st["rope_keys"]


def _prompt(st):
    d = st["case"]["dim"]
    k, v = st["kv"][..., :d], st["kv"][..., d:]
    scale = (d + ROPE) ** -0.5
    if own:
        import paper_2609_36899_amd as P
        return P.latent_prompt_attention(st["q"], k, st["rope_keys"], v, st["starts"],
                                         st["key_starts"], st["out"], scale)
    qs, ks = st["host_starts"], st["host_ends"]
    for a, b, c, e in zip(qs, qs[1:], ks, ks[1:]):
        q = st["q"][a:b].float().transpose(0, 1)
        s = torch.matmul(q[..., :d], k[c:e].float().permute(1, 2, 0))
        s = s + torch.matmul(q[..., d:], st["rope_keys"][c:e].float().t())
        last = (e - c) - (b - a) + torch.arange(b - a, device=DEV)
        hidden = torch.arange(e - c, device=DEV)[None, :] > last[:, None]
        s = (s * scale).masked_fill(hidden, -math.inf)
        out = _softmax_mix(s, v[c:e].float().transpose(0, 1))
        st["out"][a:b] = out.transpose(0, 1).to(torch.bfloat16)
    return st["out"]


def _copy(st):
    pools = [st["pages"]] + ([] if st["scales"] is None else [st["scales"]])
    if own:
        import paper_2609_36899_amd as P
        P.paged_copy_pages(pools, st["src"], st["dst"])
    else:
        src, dst = st["src"].long(), st["dst"].long()
        for pool in pools:
            pool[dst] = pool[src]
    latents, keys = _parts(st)
    return {"latents": latents, "rope_keys": keys, "scales": st["scales"]}


# ---- the definitions in 64 bits, one trajectory at a time -------------------------

def _e4m3(code):
    """The value of each E4M3 code, from its fields."""
    c = code.long()
    sign = 1.0 - 2.0 * (c >> 7).double()
    e, m = (c >> 3) & 15, (c & 7).double()
    return sign * torch.where(e > 0, (1 + m / 8) * torch.exp2(e.double() - 7), m / 512)


def _held(st, ids):
    """Latents and rotary keys of the tokens of pages `ids`, in order."""
    r = st["case"]["latent"]
    p = st["pages"][ids]
    if st["scales"] is None:
        p = p.double().flatten(0, 1)
        return p[:, :r], p[:, r:]
    c = _e4m3(p[..., :r]) * st["scales"][ids].double()[..., None]
    bits = p[..., r:].reshape(-1, ROPE, 2).int()
    k = ((bits[..., 1] << 24) | (bits[..., 0] << 16)).view(torch.float32).double()
    return c.flatten(0, 1), k


def _mix64(q, k, v, limits, scale):
    """softmax(scale q k^T) v, row i over the first limits[i] keys; limits are 1 or more."""
    s = (q @ k.T) * scale
    s[torch.arange(k.shape[0], device=DEV)[None, :] >= limits[:, None]] = -math.inf
    w = torch.exp(s - s.max(dim=1, keepdim=True).values)
    return (w @ v) / w.sum(dim=1, keepdim=True)


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    if kind == "append":
        return _append64(case, st)
    if kind == "copy":
        dst, src = st["dst"].tolist(), st["src"].tolist()
        where = list(range(st["pages"].shape[0]))
        for a, b in zip(dst, src):
            where[a] = b
        latents, keys = _held_pool(st, torch.tensor(where, device=DEV))
        scales = None if st["scales"] is None else st["scales"][where].double()
        return {"latents": latents, "rope_keys": keys, "scales": scales}
    if kind == "rows":
        c, k = [], []
        for b, n in enumerate(st["host_lens"]):
            x, y = _held(st, st["table"][b, :_pages(n)].long())
            c.append(x[:n])
            k.append(y[:n])
        return torch.cat(c), torch.cat(k)
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    if kind == "attention":
        nq, heads, r = case["nq"], case["heads"], case["latent"]
        for b, n in enumerate(st["host_lens"]):
            c, k = _held(st, st["table"][b, :_pages(n)].long())
            c = c[:n]
            k = torch.cat([c, k[:n]], dim=1)
            for j in range(nq):
                m = n - nq + j + 1
                if m > 0:
                    lim = torch.full((heads,), m, device=DEV)
                    out[b, j] = _mix64(st["q"][b, j].double(), k, c, lim, 192.0 ** -0.5)
        return out
    d, qs, ks = case["dim"], st["host_starts"], st["host_ends"]
    for a, b, c, e in zip(qs, qs[1:], ks, ks[1:]):
        lim = (e - c) - (b - a) + 1 + torch.arange(b - a, device=DEV)
        shared = st["rope_keys"][c:e].double()
        for h in range(case["heads"]):
            k = torch.cat([st["kv"][c:e, h, :d].double(), shared], dim=1)
            out[a:b, h] = _mix64(st["q"][a:b, h].double(), k, st["kv"][c:e, h, d:].double(), lim,
                                 1.0 / math.sqrt(d + ROPE))
    return out


def _held_pool(st, where):
    """What the pages show, each place holding page where[place]: codes' own values."""
    r, p = st["case"]["latent"], st["pages"][where]
    if st["scales"] is None:
        p = p.double()
        return p[..., :r], p[..., r:]
    bits = p[..., r:].reshape(*p.shape[:2], ROPE, 2).int()
    k = ((bits[..., 1] << 24) | (bits[..., 0] << 16)).view(torch.float32).double()
    return _e4m3(p[..., :r]), k


def _append64(case, st):
    r, n = case["latent"], st["x"].shape[0]
    latents, keys = _held_pool(st, torch.arange(st["pages"].shape[0], device=DEV))
    scales = None if st["scales"] is None else st["scales"].double()
    starts = st["host_starts"]
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=DEV),
                                  torch.tensor(np.diff(starts), device=DEV))
    pos = torch.cat([torch.arange(m - (b - a), m, device=DEV)
                     for m, a, b in zip(st["host_lens"], starts, starts[1:])])
    page = st["table"].long()[seq, torch.div(pos, PAGE, rounding_mode="floor")]
    slot = torch.remainder(pos, PAGE)
    turn = torch.view_as_complex(st["rope"].double()[pos].contiguous())

    def rotate(x, t):
        x = x.double()
        if case["interleaved"]:
            z = torch.view_as_complex(x.reshape(*x.shape[:-1], ROPE // 2, 2).contiguous()) * t
            return torch.view_as_real(z).flatten(-2)
        z = torch.complex(*x.reshape(*x.shape[:-1], 2, ROPE // 2).unbind(-2)) * t
        return torch.cat([z.real, z.imag], dim=-1)

    x = st["x"][:, :r].double()
    c = x / torch.sqrt(x.square().sum(1, keepdim=True) / r + EPS) * st["gain"].double()
    if scales is not None:
        scale = torch.exp2(torch.ceil(torch.log2(c.abs().amax(1) / 448.0)).clamp(-100, 100))
        c = c / scale[:, None]
        scales[page, slot] = scale
    latents[page, slot] = c
    keys[page, slot] = rotate(st["x"][:, r:], turn)
    return {"q": rotate(st["heads"][..., 128:], turn[:, None]), "latents": latents,
            "rope_keys": keys, "scales": scales}
