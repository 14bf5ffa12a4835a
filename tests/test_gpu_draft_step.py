"""The operators as one decode loop uses them: every step appends a sequence's last token
and its drafts, attends to them (all pages, then the selected ones), makes logits through
the library's projection and verifies the drafts; refused drafts are taken back by the
length alone and their slots written again in the next step.  All on one stream, with no
wait between the calls.

The reference keeps the accepted tokens' keys and values in a plain array, so it knows
nothing of pages.  bf16 pages and outputs: keys, values, queries and outputs are off by
half a bf16 step each (2^-8 relative); a score of n = Dh products moves by at most
2 * 2^-8 * sum |q k| / sqrt(Dh) (q and k), weights by twice that (element and sum), and the
weights and V are rounded once each, the output once.
"""

import numpy as np
import pytest
import torch

from oracle import operators as oo
from oracle.fp8 import e4m3_decode

pytestmark = pytest.mark.gpu

HQ, HKV, DH, T, V, D = 8, 2, 64, 3, 512, 128


@pytest.mark.parametrize("fp8", [False, True])
def test_decode_loop_with_drafts(fp8):
    import paper_2609_36899_amd as P
    rng = np.random.default_rng(1)
    B, stride = 3, 12
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(s, device="cuda", generator=g)
    emb = (rand(V, D) * 0.5).to(torch.bfloat16)
    w_qkv = P.pack_weight((rand((HQ + 2 * HKV) * DH, D) * 0.1).to(torch.bfloat16))
    w_out = P.pack_weight((rand(V, HQ * DH) * 0.3).to(torch.bfloat16))
    pool = B * stride
    kt = torch.uint8 if fp8 else torch.bfloat16
    kp = torch.zeros((pool, HKV, 16, DH), dtype=kt, device="cuda")
    vp = torch.zeros((pool, HKV, DH, 16), dtype=kt, device="cuda")
    ks, vs = (torch.ones((pool, HKV), device="cuda") if fp8 else None for _ in range(2))
    means = torch.zeros((pool, HKV, DH), dtype=torch.bfloat16, device="cuda")
    table = torch.from_numpy(rng.permutation(pool).reshape(B, stride).astype(np.int32)).cuda()
    rope = P.rope_table(stride * 16, DH)
    cs = rope.cpu().numpy().astype(np.float64)
    starts = torch.arange(0, B * (T + 1) + 1, T + 1, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    tokens = torch.randint(0, V, (B, 1), device="cuda", generator=g, dtype=torch.int32)
    history = [[] for _ in range(B)]  # (k rotated, v) of accepted tokens, fp64

    for step in range(14):
        drafts = torch.randint(0, V, (B, T), device="cuda", generator=g, dtype=torch.int32)
        rows = torch.cat([tokens, drafts], 1)
        x = emb[rows.long().reshape(-1)].contiguous()
        qkv = torch.empty((B * (T + 1), w_qkv.n), device="cuda")
        P.weight_projection(x, w_qkv, qkv)
        cut = lambda a, n: qkv[:, a * DH:(a + n) * DH].unflatten(1, (n, DH))
        q, k, v = cut(0, HQ), cut(HQ, HKV), cut(HQ + HKV, HKV)
        q_out = torch.empty((B * (T + 1), HQ, DH), dtype=torch.bfloat16, device="cuda")
        lens += T + 1
        P.paged_kv_append(k, v, lens, starts, table, rope, kp, vp, k_scales=ks, v_scales=vs,
                          k_means=means, q=q, q_out=q_out)
        q4 = q_out.view(B, T + 1, HQ, DH)
        out = torch.empty_like(q4)
        P.paged_token_attention(q4, kp, vp, table, lens, out, k_scales=ks, v_scales=vs)
        last = q4[:, T].contiguous()
        chosen = torch.empty((B, HKV, 3), dtype=torch.int32, device="cuda")
        few = torch.empty_like(last)
        P.paged_select(last, means, table, lens, chosen)
        P.paged_token_attention(last, kp, vp, table, lens, few, k_scales=ks, v_scales=vs,
                                selected=chosen)
        logits = torch.empty((B * (T + 1), V), device="cuda")
        P.weight_projection(out.view(B * (T + 1), -1), w_out, logits)
        u = torch.rand((B, T + 1), device="cuda", generator=g)
        if step % 2:
            u[:, :step % T] = 0.0  # a uniform of 0 accepts any draft that has mass
        new, n = (torch.empty((B, T + 1), dtype=torch.int32, device="cuda"),
                  torch.empty(B, dtype=torch.int32, device="cuda"))
        P.verify_drafts(logits.view(B, T + 1, V), drafts, u, new, n, temperature=0.7)
        torch.cuda.synchronize()

        # -- the same from the plain history
        f64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        hk, hv, hq = f64(k), f64(v), f64(q)
        for b in range(B):
            base = len(history[b])
            assert int(lens[b]) == base + T + 1
            mine = []
            for j in range(T + 1):
                r = b * (T + 1) + j
                mine.append((oo.rotate(hk[r], cs[base + j]), hv[r]))
                qr = oo.rotate(hq[r], cs[base + j])
                keys = history[b] + mine
                for h in range(HQ):
                    kk = np.stack([e[0][h // (HQ // HKV)] for e in keys])
                    vv = np.stack([e[1][h // (HQ // HKV)] for e in keys])
                    ref, size = oo.mix(qr[h], kk, vv)
                    move = (np.abs(kk) @ np.abs(qr[h])).max() / np.sqrt(DH)
                    half = 2.0 ** -8
                    if not fp8:
                        tol = (np.expm1(4 * half * move) + 2.5 * half) * size + half * np.abs(ref)
                        got = f64(out[b, j, h])
                        assert (np.abs(got - ref) <= tol + 1e-6).all(), (step, b, j, h)
            history[b] += mine[:1 + int(n[b])]
        # attention against the pages as they are: the oracle reads what the kernels read
        dec = (lambda p, s: e4m3_decode(p.cpu().numpy()) * s.cpu().numpy()[:, :, None, None]) \
            if fp8 else (lambda p, s: f64(p))
        ref, size = oo.token_attention(f64(q4), dec(kp, ks), dec(vp, vs), table.cpu().numpy(),
                                       lens.cpu().numpy())
        tol = 1.02 * 2.0 ** -8 * size + 2.0 ** -8 * np.abs(ref) + 1e-6
        assert (np.abs(f64(out) - ref) <= tol).all()
        want = oo.select_pages(f64(last), f64(means), table.cpu().numpy(), lens.cpu().numpy(), 3)
        np.testing.assert_array_equal(chosen.cpu().numpy(), want)
        ref, size = oo.token_attention(f64(last)[:, None], dec(kp, ks), dec(vp, vs),
                                       table.cpu().numpy(), lens.cpu().numpy(), want)
        tol = 1.02 * 2.0 ** -8 * size + 2.0 ** -8 * np.abs(ref) + 1e-6
        assert (np.abs(f64(few)[:, None] - ref) <= tol).all()
        vt, vn = oo.verify_drafts(logits.view(B, T + 1, V).cpu().numpy(), None,
                                  drafts.cpu().numpy(), u.cpu().numpy(), 0.7)
        np.testing.assert_array_equal(new.cpu().numpy(), vt)
        np.testing.assert_array_equal(n.cpu().numpy(), vn)
        # Refused drafts go by the length; their slots are written again.
        lens -= T - n
        tokens = new[torch.arange(B), n.long()][:, None].contiguous()


def test_binding_refuses_wrong_tensors():
    import paper_2609_36899_amd as P
    from paper_2609_36899_amd import PdecError
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    new = lambda dt, *s: torch.zeros(s, dtype=dt, device="cuda")
    kp, vp = new(bf, 3, 2, 16, 64), new(bf, 3, 2, 64, 16)
    c8, v8, sc = new(torch.uint8, 3, 2, 16, 64), new(torch.uint8, 3, 2, 64, 16), new(f32, 3, 2)
    q, bt, lens, out = new(bf, 2, 4, 64), new(i32, 2, 3), new(i32, 2), new(bf, 2, 4, 64)
    good = dict(q=q, k_pages=kp, v_pages=vp, block_table=bt, lens=lens, out=out)
    P.paged_token_attention(**good)
    for change, word in [
            (dict(q=q.float()), "q must be"), (dict(q=q[:, :3]), "contiguous|multiple"),
            (dict(q=None), "GPU tensor"), (dict(out=new(bf, 2, 4, 128)), "out must have shape"),
            (dict(lens=lens.long()), "lens must be"), (dict(lens=lens.cpu()), "GPU tensor"),
            (dict(lens=new(i32, 3)), "lens must have"), (dict(block_table=bt.t()), "block_table"),
            (dict(v_pages=kp), "v_pages must have"), (dict(k_pages=kp.float()), "v_pages must be"),
            (dict(k_pages=kp[:, :, :8]), "16 tokens"), (dict(k_pages=c8, v_pages=v8), "k_scales"),
            (dict(k_scales=sc), "others none"),
            (dict(k_pages=c8, v_pages=v8, k_scales=sc, v_scales=new(f32, 2, 2)), "v_scales"),
            (dict(selected=new(i32, 2, 2, 5).long()), "selected"),
            (dict(q=new(bf, 2, 3, 4, 64), out=new(bf, 2, 3, 4, 64), selected=new(i32, 2, 2, 5)),
             "one query token"),
            (dict(workspace=new(torch.uint8, 16), block_table=new(i32, 2, 300)), "too small"),
            (dict(workspace=torch.zeros(1 << 20)), "workspace must be"),
            (dict(q=new(bf, 2 * 4 * 64 + 1)[1:].view(2, 4, 64)), "aligned")]:
        with pytest.raises(PdecError, match=word):
            P.paged_token_attention(**{**good, **change})
    k, rope, starts = new(bf, 5, 2, 64), P.rope_table(40, 64), new(i32, 3)
    append = dict(k=k, v=k, lens=lens, row_start=starts, block_table=bt, rope=rope, k_pages=kp,
                  v_pages=vp)
    P.paged_kv_append(**append)
    for change, word in [
            (dict(k=k.float()), "v must be"), (dict(v=new(bf, 4, 2, 64)), "v must have"),
            (dict(k=k.transpose(0, 1).contiguous().transpose(0, 1), v=k), "side by side"),
            (dict(k=k.half(), v=k.half()), "k must be"), (dict(row_start=lens), "row_start"),
            (dict(rope=rope[:, :16]), "rope"), (dict(q=k), "q_out"), (dict(q_out=k), "together"),
            (dict(k_means=new(f32, 3, 2, 64)), "k_means"), (dict(k_pages=kp.float()), "v_pages")]:
        with pytest.raises(PdecError, match=word):
            P.paged_kv_append(**{**append, **change})
    means, sel = new(bf, 3, 2, 64), new(i32, 2, 2, 3)
    P.paged_select(q, means, bt, lens, sel)
    for args, word in [((q, means.float(), bt, lens, sel), "k_means"),
                       ((q, means, bt, lens, sel[:1]), "selected"),
                       ((new(bf, 2, 3, 64), means, bt, lens, sel), "multiple"),
                       ((q, means, bt[:1], lens, sel), "block_table")]:
        with pytest.raises(PdecError, match=word):
            P.paged_select(*args)
    with pytest.raises(PdecError, match="keep_first"):
        P.paged_select(q, means, bt, lens, sel, keep_first=3)
    z, u, n = new(f32, 2, 4, 50), new(f32, 2, 4), new(i32, 2)
    verify = dict(target_logits=z, draft_tokens=new(i32, 2, 3), uniforms=u,
                  tokens_out=new(i32, 2, 4), accepted_out=n)
    P.verify_drafts(**verify)
    for change, word in [(dict(target_logits=z.double()), "target_logits"),
                         (dict(draft_tokens=new(i32, 2, 4)), "draft_tokens"),
                         (dict(draft_logits=z), "draft_logits"), (dict(temperature=0.0), "temp"),
                         (dict(uniforms=u[:, :3]), "uniforms")]:
        with pytest.raises(PdecError, match=word):
            P.verify_drafts(**{**verify, **change})
    torch.cuda.synchronize()
