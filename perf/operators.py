"""Operators of a decode step over a caller's paged KV cache, and what they are measured on.

Four kinds of case, each through the package's public entry points:

  append     paged_kv_append: new keys, rotated at their positions, and values into
             their page slots, the queries rotated on the way
  attention  paged_token_attention: one or several query tokens per trajectory over bf16
             pages, or over E4M3 pages with a scale for each page and KV head
  sparse     paged_select, then paged_token_attention over the pages it selected
  verify     verify_drafts: drafted tokens against the target's probabilities

`run` computes them in plain torch operations, or, with `own`, through the package.

Pages hold 16 tokens: K [page][kv head][16][dim], V transposed [page][kv head][dim][16].
A scaled page reads back as code * scale, the scale a power of two chosen by the page's
largest element so that it fits E4M3's 448.
"""

import math

import numpy as np
import torch

own = False

PAGE = 16
DEV = "cuda"
F8 = torch.float8_e4m3fn


def listed():
    return [
        # One token for each trajectory of a decode batch, 8-bit pages of which most are
        # part full, with the page means that page selection reads.
        dict(name="append_decode_fp8_b64", kind="append", pages="fp8", src="bf16", means=True,
             batch=64, hq=32, hkv=8, dh=128, lo=1024, hi=8192, new_lo=1, new_hi=1, draw_seed=1),
        # A prompt in one pass, straight from the q|k|v projection's fp32 output.
        dict(name="append_prompt_bf16_4096", kind="append", pages="bf16", src="f32", means=False,
             batch=1, hq=32, hkv=8, dh=128, lo=0, hi=0, new_lo=4096, new_hi=4096, draw_seed=1),
        # Tool outputs appended to four trajectories that end inside a page.
        dict(name="append_turns_fp8_b4", kind="append", pages="fp8", src="f32", means=True,
             batch=4, hq=32, hkv=8, dh=128, lo=1000, hi=6000, new_lo=100, new_hi=700,
             draw_seed=2),
        # The smallest decode call: a few short trajectories, latency alone.
        dict(name="attention_fp8_b4_short", kind="attention", pages="fp8", batch=4, hq=4, hkv=2,
             dh=64, nq=1, lo=1, hi=128, draw_seed=1),
        # A mid-sized decode batch over 8-bit pages.
        dict(name="attention_fp8_b64", kind="attention", pages="fp8", batch=64, hq=32, hkv=8,
             dh=128, nq=1, lo=1024, hi=8192, draw_seed=21),
        # Few very long contexts, each with its last token and four drafted ones.
        dict(name="attention_fp8_b8_long_nq5", kind="attention", pages="fp8", batch=8, hq=32,
             hkv=8, dh=128, nq=5, lo=65536, hi=131072, draw_seed=3),
        # Drafted tokens over bf16 pages, groups of five heads.
        dict(name="attention_bf16_b16_nq4", kind="attention", pages="bf16", batch=16, hq=40,
             hkv=8, dh=128, nq=4, lo=1024, hi=16384, draw_seed=5),
        # One very long context, 64 pages of it read.
        dict(name="sparse_bf16_b1_long", kind="sparse", pages="bf16", batch=1, hq=32, hkv=8,
             dh=128, top=64, lo=131000, hi=131000, draw_seed=7),
        # A batch of long contexts over 8-bit pages.
        dict(name="sparse_fp8_b64", kind="sparse", pages="fp8", batch=64, hq=32, hkv=8, dh=128,
             top=128, lo=8192, hi=32768, draw_seed=8),
        # One trajectory's drafts from a lookup, which gives tokens without probabilities.
        dict(name="verify_b1_lookup", kind="verify", batch=1, drafts=3, vocab=32003,
             temperature=1.0, drafter=False, std=3.0, draw_seed=1),
        # A mid-sized batch, drafts from a lookup, the larger vocabulary.
        dict(name="verify_b16_lookup", kind="verify", batch=16, drafts=8, vocab=151936,
             temperature=0.8, drafter=False, std=3.0, draw_seed=2),
        # A decode batch with a drafting model's logits beside the target's.
        dict(name="verify_b64_drafter", kind="verify", batch=64, drafts=4, vocab=128256,
             temperature=0.8, drafter=True, std=3.0, draw_seed=3),
    ]


def _log_int(rng, lo, hi):
    return int(round(float(lo) * (float(hi) / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "sparse", "verify"])
    seed = rng.randrange(1 << 20)
    hkv, group = rng.choice([(8, 4), (8, 4), (8, 5), (8, 8), (2, 2), (4, 3), (1, 16), (5, 1)])
    dh = rng.choice([128, 128, 64])
    heads = dict(hq=hkv * group, hkv=hkv, dh=dh)
    if kind == "append":
        pages = rng.choice(["fp8", "fp8", "bf16", "f32"])
        batch = _log_int(rng, 1, 128)
        new = _log_int(rng, 1, max(2, 4000 // batch)) if rng.random() < 0.6 else 1
        return dict(kind=kind, pages=pages,
                    src="f32" if pages == "f32" else rng.choice(["bf16", "f32"]),
                    means=pages != "f32" and rng.random() < 0.7, batch=batch, **heads, lo=0,
                    hi=_log_int(rng, 16, 8192), new_lo=max(1, new // 4), new_hi=new,
                    draw_seed=seed)
    if kind == "attention":
        batch, nq = _log_int(rng, 1, 96), rng.choice([1, 1, 2, 3, 5, 8, 13])
        hi = min(131072, _log_int(rng, 64, 400000 // batch))
        return dict(kind=kind, pages=rng.choice(["fp8", "fp8", "bf16"]), batch=batch, **heads,
                    nq=nq, lo=max(1, hi // rng.choice([1, 2, 8, 64])), hi=hi, draw_seed=seed)
    if kind == "sparse":
        batch = _log_int(rng, 1, 64)
        hi = min(131072, _log_int(rng, 256, 800000 // batch))
        return dict(kind=kind, pages=rng.choice(["fp8", "bf16"]), batch=batch, **heads,
                    top=rng.choice([3, 16, 33, 64, 128, 200]),
                    lo=max(1, hi // rng.choice([1, 4, 64])), hi=hi, draw_seed=seed)
    return dict(kind=kind, batch=_log_int(rng, 1, 64), drafts=rng.choice([1, 2, 3, 4, 5]),
                vocab=rng.choice([128256, 151936, 32003, 1024]),
                temperature=rng.choice([0.6, 0.8, 1.0, 1.3]), drafter=rng.random() < 0.5,
                std=rng.choice([1.0, 3.0]), draw_seed=seed)


# ---- sizes that follow from a case alone ------------------------------------

def _pages(n):
    return (n + PAGE - 1) // PAGE


def _lens(case):
    """Cached tokens of each trajectory, the new ones among them, and the new ones."""
    rng = np.random.default_rng(case["draw_seed"])
    ctx = rng.integers(case["lo"], case["hi"] + 1, size=case["batch"])
    if case["kind"] == "append":
        new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["batch"])
        return ctx + new, new
    return ctx, None


def work(case):
    kind = case["kind"]
    if kind == "verify":
        rows = case["batch"] * (case["drafts"] + 1 + (case["drafts"] if case["drafter"] else 0))
        return {"bytes": rows * case["vocab"] * 4, "flops": rows * case["vocab"] * 4}
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    lens, new = _lens(case)
    el = {"fp8": 1, "bf16": 2, "f32": 4}[case["pages"]]
    if kind == "append":
        n = int(new.sum())
        src = 2 if case["src"] == "bf16" else 4
        by = n * (hq + 2 * hkv) * dh * src                       # q, k, v in
        by += n * hq * dh * (4 if case["pages"] == "f32" else 2)  # q out
        by += n * 2 * hkv * dh * el                              # page slots
        by += n * dh * 4                                         # rotation table
        touched = int((_pages(lens) - (lens - new) // PAGE).sum())
        old = int(((lens - new) % PAGE).sum())                   # tokens before, in those pages
        if case["pages"] == "fp8":
            by += touched * hkv * 16                             # scales in and out
        if case["means"]:
            by += touched * hkv * dh * 2 + old * hkv * dh * el
        return {"bytes": by, "flops": n * (hq + hkv) * dh * 3}
    if kind == "attention":
        nq, keys = case["nq"], int(lens.sum())
        by = keys * 2 * hkv * dh * el + 2 * case["batch"] * nq * hq * dh * 2
        if case["pages"] == "fp8":
            by += int(_pages(lens).sum()) * hkv * 8
        return {"bytes": by, "flops": 4 * keys * nq * hq * dh}
    n_pages = _pages(lens)
    taken = np.minimum(n_pages, case["top"])
    by = int(n_pages.sum()) * hkv * dh * 2                       # page means
    by += int(taken.sum()) * hkv * (2 * PAGE * dh * el + 4 + (8 if case["pages"] == "fp8" else 0))
    by += 2 * case["batch"] * hq * dh * 2
    return {"bytes": by, "flops": 2 * int(n_pages.sum()) * hq * dh
            + 4 * int(taken.sum()) * PAGE * hq * dh}


# ---- inputs ------------------------------------------------------------------

def _rope_table(max_pos, dh):
    """(cos, sin) of each position and pair, angles in 64 bits."""
    inv = 10000.0 ** (-2.0 * torch.arange(dh // 2, dtype=torch.float64, device=DEV) / dh)
    ang = torch.arange(max_pos, dtype=torch.float64, device=DEV)[:, None] * inv
    return torch.stack([ang.cos(), ang.sin()], dim=-1).float().contiguous()


def _codes(g, shape):
    """E4M3 codes as a page scaled to its largest element holds them (a deviation of 100)."""
    x = torch.randn(shape, dtype=torch.bfloat16, device=DEV, generator=g)
    return x.mul_(100.0).clamp_(-448.0, 448.0).to(F8).view(torch.uint8)


def _scales(g, shape):
    e = torch.randint(-8, -5, shape, device=DEV, generator=g)
    return torch.exp2(e.float())


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind = case["kind"]
    if kind == "verify":
        B, T, V = case["batch"], case["drafts"], case["vocab"]
        target = torch.randn((B, T + 1, V), device=DEV, generator=g).mul_(case["std"])
        st = dict(case=case, target=target, drafter=None)
        if case["drafter"]:
            # A drafting model's logits: the target's with an error of their own, and
            # tokens drawn from them (the largest of logits plus Gumbel noise).
            d = target[:, :T].contiguous()
            d.add_(torch.randn(d.shape, device=DEV, generator=g))
            st["drafter"] = d
            like = d
        else:
            like = target[:, :T]
        u = torch.rand(like.shape, device=DEV, generator=g).clamp_min_(1e-20)
        st["drafts"] = (like / case["temperature"] - torch.log(-torch.log(u))).argmax(-1).int()
        if not case["drafter"]:
            # What a lookup finds is often right: its tokens get about half of the mass.
            all_ = torch.logsumexp(like / case["temperature"], -1, keepdim=True)
            target[:, :T].scatter_(2, st["drafts"][..., None].long(), all_ * case["temperature"])
        st["u"] = torch.rand((B, T + 1), device=DEV, generator=g)
        st["tokens"] = torch.empty((B, T + 1), dtype=torch.int32, device=DEV)
        st["accepted"] = torch.empty(B, dtype=torch.int32, device=DEV)
        return st

    hq, hkv, dh, B = case["hq"], case["hkv"], case["dh"], case["batch"]
    lens, new = _lens(case)
    n_pages = _pages(lens)
    pool = int(n_pages.sum()) + 3
    perm = torch.randperm(pool, device=DEV, generator=g).int()
    stride = int(n_pages.max()) + 1
    at = np.concatenate([[0], np.cumsum(n_pages)[:-1]])[:, None] + np.arange(stride)[None]
    used = np.arange(stride)[None] < n_pages[:, None]
    at = torch.from_numpy(np.where(used, at, 0)).to(DEV)
    table = torch.where(torch.from_numpy(used).to(DEV), perm[at], torch.zeros_like(perm[:1]))
    st = dict(case=case, table=table.contiguous(),
              lens=torch.from_numpy(lens.astype(np.int32)).to(DEV), ks=None, vs=None, means=None)
    kshape, vshape = (pool, hkv, PAGE, dh), (pool, hkv, dh, PAGE)
    if case["pages"] == "fp8":
        st["k"], st["v"] = _codes(g, kshape), _codes(g, vshape)
        st["ks"], st["vs"] = _scales(g, (pool, hkv)), _scales(g, (pool, hkv))
    else:
        td = torch.bfloat16 if case["pages"] == "bf16" else torch.float32
        st["k"] = torch.randn(kshape, dtype=td, device=DEV, generator=g)
        st["v"] = torch.randn(vshape, dtype=td, device=DEV, generator=g)
    qt = torch.float32 if case["pages"] == "f32" else torch.bfloat16

    if kind == "append":
        n = int(new.sum())
        st["rope"] = _rope_table(int(lens.max()), dh)
        td = torch.bfloat16 if case["src"] == "bf16" else torch.float32
        st["qkv"] = torch.randn((n, hq + 2 * hkv, dh), dtype=td, device=DEV, generator=g)
        # Keys whose size differs from token to token, so that appended tokens outgrow a
        # part-full page's scale now and then.
        size = torch.exp2(torch.randn((n, 1, 1), device=DEV, generator=g)).to(td)
        st["qkv"][:, hq:].mul_(size)
        starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        st["starts"] = torch.from_numpy(starts).to(DEV)
        # Rows that are the first of the call in their page, known where the call is planned.
        first = np.concatenate([(np.arange(a - m, a) % PAGE == 0) | (np.arange(m) == 0)
                                for a, m in zip(lens, new)])
        st["leaders"] = torch.from_numpy(np.nonzero(first)[0]).to(DEV)
        st["q_out"] = torch.empty((n, hq, dh), dtype=qt, device=DEV)
        if case["means"]:
            st["means"] = torch.zeros((pool, hkv, dh), dtype=torch.bfloat16, device=DEV)
        return st

    if kind == "attention":
        shape = (B, case["nq"], hq, dh)
    else:
        shape = (B, hq, dh)
        # Means of 16 keys of deviation 0.8 apiece, some pages nearer to the query than others.
        m = torch.randn((pool, hkv, dh), device=DEV, generator=g) * 0.2
        m *= torch.exp2(0.5 * torch.randn((pool, hkv, 1), device=DEV, generator=g))
        st["means"] = m.to(torch.bfloat16)
        st["selected"] = torch.empty((B, hkv, case["top"]), dtype=torch.int32, device=DEV)
    st["q"] = torch.randn(shape, dtype=torch.bfloat16, device=DEV, generator=g)
    st["out"] = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    return st


# ---- one pass ------------------------------------------------------------------

def run(state):
    return {"append": _append, "attention": _attention, "sparse": _sparse,
            "verify": _verify}[state["case"]["kind"]](state)


def _append(st):
    case = st["case"]
    hq, hkv = case["hq"], case["hkv"]
    q, k, v = st["qkv"][:, :hq], st["qkv"][:, hq:hq + hkv], st["qkv"][:, hq + hkv:]
    if own:
        import paper_2609_36899_amd as P
        P.paged_kv_append(k, v, st["lens"], st["starts"], st["table"], st["rope"], st["k"],
                          st["v"], k_scales=st["ks"], v_scales=st["vs"], k_means=st["means"],
                          q=q, q_out=st["q_out"])
    else:
        _append_plain(st, q, k, v)
    fp8 = case["pages"] == "fp8"
    return {"q": st["q_out"], "k": st["k"].view(F8) if fp8 else st["k"],
            "v": st["v"].view(F8) if fp8 else st["v"], "k_scales": st["ks"],
            "v_scales": st["vs"], "means": st["means"]}


def _rotate(x, cs):
    half = x.shape[-1] // 2
    a, b = x[..., :half].float(), x[..., half:].float()
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    return torch.cat([a * c - b * s, a * s + b * c], dim=-1)


def _scale_for(amax):
    """The smallest power of two that brings amax to 448 or less."""
    m, e = torch.frexp(amax)
    e = e - 9 + (m > 0.875).int()
    e = torch.where(amax > 0, e, torch.full_like(e, -100)).clamp(-100, 100)
    return torch.ldexp(torch.ones_like(amax), e)


def _append_plain(st, q, k, v):
    case = st["case"]
    starts, lens, lead = st["starts"].long(), st["lens"].long(), st["leaders"]
    r = torch.arange(k.shape[0], device=DEV)
    seq = torch.searchsorted(starts[1:], r, right=True)
    pos = lens[seq] - (starts[seq + 1] - r)
    page, slot = st["table"][seq, pos // PAGE].long(), pos % PAGE
    cs = st["rope"][pos]
    st["q_out"].copy_(_rotate(q, cs))
    k, v = _rotate(k, cs), v.float()
    lp, lslot = page[lead], slot[lead]
    before = torch.arange(PAGE, device=DEV)[None, :] < lslot[:, None]  # slots filled earlier
    if case["pages"] == "fp8":
        owner = torch.searchsorted(lead, r, right=True) - 1
        for x, pages, scales, token_axis in ((k, st["k"], st["ks"], 2), (v, st["v"], st["vs"], 3)):
            amax = torch.zeros((lp.shape[0], x.shape[1]), device=DEV)
            amax.scatter_reduce_(0, owner[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
            need, old = _scale_for(amax), scales[lp]
            scale = torch.where((lslot == 0)[:, None], need, torch.maximum(old, need))
            had = pages[lp]
            moved = had.view(F8).float() * old[:, :, None, None] / scale[:, :, None, None]
            keep = before[:, None, :, None] if token_axis == 2 else before[:, None, None, :]
            pages[lp] = torch.where(keep, moved.clamp(-448, 448).to(F8).view(torch.uint8), had)
            scales[lp] = scale
            codes = (x / scale[owner][:, :, None]).clamp(-448, 448).to(F8).view(torch.uint8)
            if token_axis == 2:
                pages[page, :, slot] = codes
            else:
                pages[page, :, :, slot] = codes
    else:
        st["k"][page, :, slot] = k.to(st["k"].dtype)
        st["v"][page, :, :, slot] = v.to(st["v"].dtype)
    if st["means"] is not None:
        n = (lens[seq][lead] - pos[lead] // PAGE * PAGE).clamp(max=PAGE)
        keys = st["k"][lp]
        keys = (keys.view(F8).float() * st["ks"][lp][:, :, None, None]
                if case["pages"] == "fp8" else keys.float())
        filled = torch.arange(PAGE, device=DEV)[None, :] < n[:, None]
        keys = torch.where(filled[:, None, :, None], keys, torch.zeros_like(keys[:1]))
        st["means"][lp] = (keys.sum(2) / n[:, None, None]).to(torch.bfloat16)


def _read(pages, scales, ids):
    """Pages `ids` in 32 bits."""
    x = pages[ids]
    if scales is None:
        return x.float()
    return x.view(F8).float() * scales[ids][..., None, None]


def _softmax_mix(q, k, v, seen):
    """q [..., R, D], k [..., L, D], v [..., D, L], seen [..., R, L]."""
    s = torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(q.shape[-1])
    s = s.masked_fill(~seen, -math.inf)
    m = s.amax(-1, keepdim=True)
    e = torch.exp(s - m.masked_fill(m == -math.inf, 0.0))
    total = e.sum(-1, keepdim=True)
    return torch.matmul(e, v.transpose(-1, -2)) / total.masked_fill(total == 0, 1.0)


def _attention(st):
    if own:
        import paper_2609_36899_amd as P
        return P.paged_token_attention(st["q"], st["k"], st["v"], st["table"], st["lens"],
                                       st["out"], k_scales=st["ks"], v_scales=st["vs"])
    case, q = st["case"], st["q"]
    B, nq, hq, dh = q.shape
    hkv = case["hkv"]
    ids = st["table"].long()
    k = _read(st["k"], st["ks"], ids).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, dh)
    v = _read(st["v"], st["vs"], ids).permute(0, 2, 3, 1, 4).reshape(B, hkv, dh, -1)
    pos = torch.arange(k.shape[2], device=DEV)
    lens = st["lens"].long()
    v = v.masked_fill((pos[None, :] >= lens[:, None])[:, None, None, :], 0.0)
    last = lens[:, None] - nq + torch.arange(nq, device=DEV)[None, :]  # a row's own position
    seen = (pos[None, None, :] <= last[:, :, None])[:, None, :, None, :]
    seen = seen.expand(B, 1, nq, hq // hkv, -1).reshape(B, 1, -1, k.shape[2])
    rows = q.float().reshape(B, nq, hkv, hq // hkv, dh).transpose(1, 2).reshape(B, hkv, -1, dh)
    out = _softmax_mix(rows, k, v, seen).reshape(B, hkv, nq, hq // hkv, dh)
    st["out"].copy_(out.transpose(1, 2).reshape(q.shape))
    return st["out"]


def _sparse(st):
    case, q = st["case"], st["q"]
    if own:
        import paper_2609_36899_amd as P
        P.paged_select(q, st["means"], st["table"], st["lens"], st["selected"])
        P.paged_token_attention(q, st["k"], st["v"], st["table"], st["lens"], st["out"],
                                k_scales=st["ks"], v_scales=st["vs"], selected=st["selected"])
        return st["selected"], st["out"]
    B, hq, dh = q.shape
    hkv, top = case["hkv"], case["top"]
    ids, lens = st["table"].long(), st["lens"].long()
    n = (lens + PAGE - 1) // PAGE
    # Scores next to the last one taken decide which page is read: 64 bits, as whole
    # numbers have to come out equal, and rounded to 32 once.
    means = st["means"][ids].double().permute(0, 2, 3, 1)
    score = torch.matmul(q.double().reshape(B, hkv, hq // hkv, dh), means).amax(2).float()
    page = torch.arange(ids.shape[1], device=DEV)
    forced = (page[None, :] == 0) | (page[None, :] == n[:, None] - 1)
    score = score.masked_fill(forced[:, None], math.inf)
    score = score.masked_fill((page[None, :] >= n[:, None])[:, None], -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :top]
    if best.shape[-1] < top:
        best = torch.nn.functional.pad(best, (0, top - best.shape[-1]), value=ids.shape[1])
    taken = torch.arange(top, device=DEV)[None, None, :] < n[:, None, None]
    best = best.masked_fill(~taken, ids.shape[1]).sort(-1).values
    st["selected"].copy_(best.masked_fill(~taken, -1))
    best = best.masked_fill(~taken, 0)
    phys = torch.gather(ids[:, None].expand(-1, hkv, -1), 2, best)
    head = torch.arange(hkv, device=DEV)[None, :, None]
    k, v = st["k"][phys, head], st["v"][phys, head]
    if st["ks"] is not None:
        k = k.view(F8).float() * st["ks"][phys, head][..., None, None]
        v = v.view(F8).float() * st["vs"][phys, head][..., None, None]
    pos = best[..., None] * PAGE + torch.arange(PAGE, device=DEV)
    seen = (pos < lens[:, None, None, None]) & taken[..., None]
    v = v.float().masked_fill(~seen[:, :, :, None, :], 0.0).permute(0, 1, 3, 2, 4)
    out = _softmax_mix(q.float().reshape(B, hkv, hq // hkv, dh),
                       k.float().reshape(B, hkv, -1, dh), v.reshape(B, hkv, dh, -1),
                       seen.reshape(B, hkv, 1, -1))
    st["out"].copy_(out.reshape(q.shape))
    return st["selected"], st["out"]


def _masses(z, temperature):
    """Whole-number masses exp((z - max z) / T) * 2^40 of each row, and their sums."""
    x = (z.double() - z.amax(-1, keepdim=True).double()) * (1.0 / float(np.float32(temperature)))
    m = torch.round(torch.exp(x) * 2.0 ** 40).long()
    return m, m.sum(-1)


def _verify(st):
    case = st["case"]
    if own:
        import paper_2609_36899_amd as P
        P.verify_drafts(st["target"], st["drafts"], st["u"], st["tokens"], st["accepted"],
                        temperature=case["temperature"], draft_logits=st["drafter"])
        return st["tokens"], st["accepted"]
    B, T = st["drafts"].shape
    x = st["drafts"].long()
    p, ps = _masses(st["target"], case["temperature"])
    pi = 2.0 ** 50 / ps.double()
    px = torch.gather(p[:, :T], 2, x[..., None])[..., 0].double() * pi[:, :T]
    u24 = torch.floor(st["u"] * 2.0 ** 24).long()
    if st["drafter"] is not None:
        d, ds = _masses(st["drafter"], case["temperature"])
        di = 2.0 ** 50 / ds.double()
        dx = torch.gather(d, 2, x[..., None])[..., 0].double() * di
    else:
        dx = torch.full_like(px, 2.0 ** 50)
    ok = u24[:, :T].double() * dx < 2.0 ** 24 * px
    n = ok.long().cumprod(1).sum(1)
    row = torch.arange(B, device=DEV)
    left = p[row, n].double() * pi[row, n][:, None]
    drafted = n < T
    at = n.clamp(max=T - 1)
    if st["drafter"] is not None:
        off = d[row, at].double() * di[row, at][:, None]
    else:
        off = torch.zeros_like(left).scatter_(1, x[row, at][:, None], math.inf)
    rest = torch.round((left - off.masked_fill(~drafted[:, None], 0.0)).clamp_min(0.0)).long()
    rest = torch.where((rest.sum(1) == 0)[:, None], torch.round(left).long(), rest)
    z = rest.sum(1)
    ul = u24[:, T]
    goal = ul * (z >> 24) + ((ul * (z & 0xFFFFFF)) >> 24)
    nxt = (rest.cumsum(1) > goal[:, None]).int().argmax(1)
    j = torch.arange(T + 1, device=DEV)[None, :]
    both = torch.cat([x, torch.full_like(x[:, :1], -1)], 1)
    both = torch.where(j < n[:, None], both, torch.full_like(both, -1))
    both = torch.where(j == n[:, None], nxt[:, None], both)
    st["tokens"].copy_(both)
    st["accepted"].copy_(n)
    return st["tokens"], st["accepted"]


# ---- the definitions in 64 bits, one trajectory at a time -------------------------

def _mix64(q, k, v):
    """softmax(q k^T / sqrt(D)) v of rows q [G, D] over keys k [L, D], values v [L, D]."""
    if k.shape[0] == 0:
        return torch.zeros_like(q)
    s = (q @ k.T) * q.shape[1] ** -0.5
    w = torch.exp(s - s.max(dim=1, keepdim=True).values)
    return (w @ v) / w.sum(dim=1, keepdim=True)


def _e4m3(code):
    """The value of each E4M3 code, from its fields."""
    c = code.long()
    sign = 1.0 - 2.0 * (c >> 7).double()
    e, m = (c >> 3) & 15, (c & 7).double()
    return sign * torch.where(e > 0, (1 + m / 8) * torch.exp2(e.double() - 7), m / 512)


def _to_e4m3(x):
    """x rounded to the nearest value of E4M3 (ties to even), at most 448 in size."""
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)
    return torch.copysign(torch.round(a / step) * step, x)


def exact(case, seed):
    if case["kind"] == "verify":
        return None
    st = prepare(case, seed)
    if case["kind"] == "append":
        return _append64(case, st)
    lens = st["lens"].tolist()
    hkv, G = case["hkv"], case["hq"] // case["hkv"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    fp8 = case["pages"] == "fp8"

    def keys(b, g, which):
        ids = st["table"][b, which].long()
        k, v = st["k"][ids, g], st["v"][ids, g]
        k, v = (_e4m3(k), _e4m3(v)) if fp8 else (k.double(), v.double())
        if fp8:
            k = k * st["ks"][ids, g].double()[:, None, None]
            v = v * st["vs"][ids, g].double()[:, None, None]
        return k.reshape(-1, case["dh"]), v.transpose(1, 2).reshape(-1, case["dh"])

    for b, n in enumerate(lens):
        np_ = (n + PAGE - 1) // PAGE
        for g in range(hkv):
            if case["kind"] == "attention":
                k, v = keys(b, g, torch.arange(np_, device=DEV))
                for j in range(case["nq"]):
                    m = max(0, n - case["nq"] + j + 1)
                    q = st["q"][b, j, g * G:(g + 1) * G].double()
                    out[b, j, g * G:(g + 1) * G] = _mix64(q, k[:m], v[:m])
                continue
            q = st["q"][b, g * G:(g + 1) * G].double()
            means = st["means"][st["table"][b, :np_].long(), g].double()
            score = (means @ q.T).max(dim=1).values.float()
            score[0] = math.inf
            score[np_ - 1] = math.inf
            which = torch.argsort(score, descending=True, stable=True)[:case["top"]].sort().values
            k, v = keys(b, g, which)
            m = k.shape[0] - (np_ * PAGE - n)
            out[b, g * G:(g + 1) * G] = _mix64(q, k[:m], v[:m])
    return out if case["kind"] == "attention" else (None, out)


def _append64(case, st):
    hq, hkv, dh = case["hq"], case["hkv"], case["dh"]
    fp8, el = case["pages"] == "fp8", torch.float64
    lens, starts = st["lens"].tolist(), st["starts"].tolist()
    x = st["qkv"].double()
    pos = torch.cat([torch.arange(n - (b - a), n) for n, a, b in zip(lens, starts, starts[1:])])
    cs = st["rope"].double()[pos.to(DEV)][:, None]
    turn = torch.view_as_complex(cs.contiguous())
    halves = x[:, :hq + hkv].reshape(x.shape[0], hq + hkv, 2, dh // 2)
    z = torch.complex(halves[:, :, 0], halves[:, :, 1]) * turn
    rot = torch.cat([z.real, z.imag], dim=-1)
    k_new, v_new = rot[:, hq:], x[:, hq + hkv:]
    k = _e4m3(st["k"]) if fp8 else st["k"].to(el)
    v = (_e4m3(st["v"]) if fp8 else st["v"].to(el)).transpose(2, 3).contiguous()
    ks = st["ks"].double() if fp8 else None
    vs = st["vs"].double() if fp8 else None
    means = st["means"].double() if st["means"] is not None else None
    for b, n in enumerate(lens):
        p = n - (starts[b + 1] - starts[b])
        while p < n:
            page = int(st["table"][b, p // PAGE])
            s0 = p % PAGE
            m = min(PAGE - s0, n - p)
            r = starts[b] + p - (n - (starts[b + 1] - starts[b]))
            for pages, scales, new in ((k, ks, k_new), (v, vs, v_new)):
                rows = new[r:r + m].transpose(0, 1)  # [head][token][dim]
                if not fp8:
                    pages[page, :, s0:s0 + m] = rows
                    continue
                top = rows.abs().amax((1, 2))
                want = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(-100, 100))
                scale = want if s0 == 0 else torch.maximum(want, scales[page])
                ratio = (scales[page] / scale)[:, None, None]
                pages[page, :, :s0] = _to_e4m3(pages[page, :, :s0] * ratio)
                pages[page, :, s0:s0 + m] = rows / scale[:, None, None]
                scales[page] = scale
            if means is not None:
                held = k[page, :, :s0 + m]
                if fp8:
                    held = _to_e4m3(held) * ks[page][:, None, None]
                else:
                    held = held.to(st["k"].dtype).double()
                means[page] = held.mean(1)
            p += m
    return {"q": rot[:, :hq], "k": k, "v": v.transpose(2, 3), "k_scales": ks, "v_scales": vs,
            "means": means}
