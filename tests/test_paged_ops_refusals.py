"""What the calls over caller-owned pages and verify_drafts refuse, on the host: no
launch is made, so made-up addresses serve as pointers."""

import pytest
import torch

from paper_2609_36899_amd import _native as N
from paper_2609_36899_amd import paged
from paper_2609_36899_amd._native import PdecError

A = 1 << 20  # a made-up, aligned address


def _append(**kw):
    a = dict(src=N.BF16, kv=N.BF16, rows=4, seqs=2, hq=4, hkv=2, dh=64, q=A, qs=256, k=A, ks=128,
             v=A, vs=128, lens=A, start=A, bt=A, stride=8, pages=9, rope=A, max_pos=50, qo=A, kp=A,
             vp=A, kscale=None, vscale=None, means=None)
    a.update(kw)
    return N.load().paged_kv_append(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(src=2), N.INVALID_ARG, b"src_dtype"), (dict(kv=3), N.INVALID_ARG, b"kv_dtype"),
    (dict(kv=N.F32), N.UNSUPPORTED, b"fp32 rows"), (dict(k=None), N.INVALID_ARG, b"null"),
    (dict(qo=None), N.INVALID_ARG, b"null"), (dict(q=None), N.INVALID_ARG, b"null"),
    (dict(lens=None), N.INVALID_ARG, b"null"), (dict(hq=5), N.INVALID_ARG, b"multiple"),
    (dict(hq=34), N.UNSUPPORTED, b"at most 16"), (dict(dh=96), N.UNSUPPORTED, b"head_dim"),
    (dict(seqs=0), N.INVALID_ARG, b"batch"), (dict(stride=0), N.INVALID_ARG, b"bt_stride"),
    (dict(stride=(1 << 22) + 1), N.INVALID_ARG, b"bt_stride"),
    (dict(pages=0), N.INVALID_ARG, b"n_pages"), (dict(pages=1 << 31), N.INVALID_ARG, b"n_pages"),
    (dict(rows=-1), N.INVALID_ARG, b"n_rows"), (dict(max_pos=0), N.INVALID_ARG, b"max_pos"),
    (dict(ks=127), N.INVALID_ARG, b"strides"), (dict(qs=255), N.INVALID_ARG, b"strides"),
    (dict(kscale=A), N.INVALID_ARG, b"scales"), (dict(kv=N.FP8_E4M3), N.INVALID_ARG, b"scales"),
    (dict(kv=N.FP8_E4M3, kscale=A), N.INVALID_ARG, b"scales"),
    (dict(src=N.F32, kv=N.F32, means=A), N.UNSUPPORTED, b"means"),
    (dict(kp=A + 8), N.INVALID_ARG, b"aligned"), (dict(rope=A + 4), N.INVALID_ARG, b"aligned"),
    (dict(rows=1 << 30), N.INVALID_ARG, b"too many rows"),
])
def test_append(kw, code, word):
    assert _append(**kw) == code
    assert word in N.load().last_error()


def test_append_of_no_rows_is_nothing():
    assert _append(rows=0) == N.OK


def _attn(**kw):
    a = dict(kv=N.BF16, batch=2, n_q=1, hq=4, hkv=2, dh=64, q=A, kp=A, vp=A, ks=None, vs=None,
             pages=9, bt=A, stride=800, lens=A, sel=None, n_sel=0, out=A, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return N.load().paged_token_attention(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(kv=N.F32), N.INVALID_ARG, b"kv_dtype"), (dict(q=None), N.INVALID_ARG, b"null"),
    (dict(ws=None), N.INVALID_ARG, b"too small"), (dict(n_q=0), N.INVALID_ARG, b"n_q"),
    (dict(n_q=4097), N.INVALID_ARG, b"n_q"), (dict(batch=0), N.INVALID_ARG, b"batch"),
    (dict(hq=3), N.INVALID_ARG, b"multiple"), (dict(hq=34), N.UNSUPPORTED, b"at most 16"),
    (dict(dh=32), N.UNSUPPORTED, b"head_dim"), (dict(vs=A), N.INVALID_ARG, b"scales"),
    (dict(kv=N.FP8_E4M3), N.INVALID_ARG, b"scales"),
    (dict(sel=A, n_sel=4, n_q=2), N.INVALID_ARG, b"one query token"),
    (dict(sel=A, n_sel=0), N.INVALID_ARG, b"n_selected"),
    (dict(out=A + 2), N.INVALID_ARG, b"aligned"), (dict(ws_bytes=100), N.INVALID_ARG, b"too small"),
    (dict(batch=1 << 20, stride=1 << 22), N.INVALID_ARG, b"too large"),
])
def test_attention(kw, code, word):
    assert _attn(**kw) == code
    assert word in N.load().last_error()


def _select(**kw):
    a = dict(batch=2, hq=4, hkv=2, dh=64, q=A, means=A, pages=9, bt=A, stride=8, lens=A, n_sel=4,
             first=1, last=1, sel=A, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return N.load().paged_select(*a.values(), None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(q=None), N.INVALID_ARG, b"null"), (dict(sel=None), N.INVALID_ARG, b"null"),
    (dict(hq=5), N.INVALID_ARG, b"multiple"), (dict(dh=80), N.UNSUPPORTED, b"head_dim"),
    (dict(n_sel=0), N.INVALID_ARG, b"n_selected"), (dict(first=-1), N.INVALID_ARG, b"keep_first"),
    (dict(last=0), N.INVALID_ARG, b"keep_last"), (dict(first=3, last=2), N.INVALID_ARG, b"at most"),
    (dict(means=A + 2), N.INVALID_ARG, b"aligned"), (dict(ws_bytes=0), N.INVALID_ARG, b"too small"),
    (dict(stride=0), N.INVALID_ARG, b"bt_stride"),
])
def test_select(kw, code, word):
    assert _select(**kw) == code
    assert word in N.load().last_error()


def _verify(**kw):
    a = dict(batch=2, n=3, vocab=100, target=A, drafter=A, drafts=A, u=A, t=1.0, tokens=A,
             accepted=A, ws=A, ws_bytes=1 << 40)
    a.update(kw)
    return N.load().verify_drafts(*a.values(), None)


@pytest.mark.parametrize("kw,word", [
    (dict(target=None), b"null"), (dict(accepted=None), b"null"), (dict(t=0.0), b"temperature"),
    (dict(t=float("inf")), b"temperature"), (dict(t=float("nan")), b"temperature"),
    (dict(batch=0), b"sizes"), (dict(n=0), b"sizes"), (dict(n=1025), b"sizes"),
    (dict(vocab=0), b"sizes"), (dict(vocab=(1 << 22) + 1), b"sizes"),
    (dict(ws_bytes=8), b"too small"), (dict(ws=A + 4), b"aligned"), (dict(target=A + 2), b"aligned"),
])
def test_verify(kw, word):
    assert _verify(**kw) == N.INVALID_ARG
    assert word in N.load().last_error()


def test_rope_table():
    lib = N.load()
    assert lib.rope_table(0, 64, 1e4, A, None) == N.INVALID_ARG
    assert lib.rope_table(8, 63, 1e4, A, None) == N.INVALID_ARG
    assert lib.rope_table(8, 64, 0.0, A, None) == N.INVALID_ARG
    assert lib.rope_table(8, 64, 1e4, None, None) == N.INVALID_ARG


def test_sizes_of_workspaces():
    lib = N.load()
    a = paged.paged_token_attention_workspace_bytes(64, 1, 32, 8, 128, 512)
    b = paged.paged_token_attention_workspace_bytes(64, 5, 32, 8, 128, 512)
    assert 0 < a < b < 1 << 30
    assert paged.paged_token_attention_workspace_bytes(64, 5, 32, 8, 128, 16) == 0
    assert paged.paged_select_workspace_bytes(2, 8, 100) >= 2 * 8 * 100 * 4
    assert paged.verify_drafts_workspace_bytes(4, 3, 32000, True) > \
        paged.verify_drafts_workspace_bytes(4, 3, 32000, False) > 0
    assert lib.paged_token_attention_workspace_bytes(0, 1, 4, 2, 64, 9) == N.INVALID_ARG
    assert lib.paged_token_attention_workspace_bytes(1, 1, 4, 2, 64, 0) == N.INVALID_ARG
    assert lib.paged_select_workspace_bytes(1, 0, 8) == N.INVALID_ARG
    assert lib.verify_drafts_workspace_bytes(1, 1, 0, 0) == N.INVALID_ARG


def test_binding_refuses_tensors_of_the_host():
    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    pages = torch.zeros((3, 2, 16, 64), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(PdecError, match="GPU"):
        paged.paged_token_attention(x, pages, pages.transpose(2, 3).contiguous(), i[:, None], i, x)
    with pytest.raises(PdecError, match="GPU"):
        paged.paged_select(x, pages[:, :, 0].contiguous(), i[:, None], i, i[:, None, None])
    with pytest.raises(PdecError, match="GPU"):
        paged.verify_drafts(torch.zeros((2, 2, 9)), i[:, None], torch.zeros((2, 2)),
                            torch.zeros((2, 2), dtype=torch.int32), i)
    with pytest.raises(PdecError, match="table size"):
        paged.rope_table(0, 64)


def test_a_workspace_of_the_largest_sizes_serves_all_smaller_ones():
    """A batch that shrinks keeps its workspace: no size asks for more than a larger one."""
    attn, verify = (paged.paged_token_attention_workspace_bytes,
                    paged.verify_drafts_workspace_bytes)
    for hq, hkv in ((32, 8), (8, 2), (16, 1), (5, 5)):
        for n_q in (1, 5, 13, 40):
            for pages in (8, 48, 49, 128, 132, 133, 4000):
                need = [attn(b, n_q, hq, hkv, 128, pages) for b in range(1, 600)]
                assert need == sorted(need), (hq, hkv, n_q, pages)
        for batch in (1, 20, 63, 64, 500):
            for pages in (48, 128, 133):
                need = [attn(batch, n, hq, hkv, 128, pages) for n in range(1, 200)]
                assert need == sorted(need), (hq, hkv, batch, pages)
            need = [attn(batch, 3, hq, hkv, 128, p) for p in range(1, 300)]
            assert need == sorted(need), (hq, hkv, batch)
    for vocab in (1, 1024, 32003, 128256, 151936):
        for drafter in (True, False):
            for n in (1, 4, 9):
                need = [verify(b, n, vocab, drafter) for b in range(1, 400)]
                assert need == sorted(need), (vocab, drafter, n)
            for batch in (1, 8, 25, 64):
                need = [verify(batch, n, vocab, drafter) for n in range(1, 60)]
                assert need == sorted(need), (vocab, drafter, batch)
        assert all(verify(b, 4, vocab, False) <= verify(b, 4, vocab, True) for b in range(1, 400))


def test_a_call_takes_the_workspace_of_a_larger_batch():
    """63 sequences in the workspace of 64: refused for nothing but the launch itself, which
    has no GPU here."""
    need = paged.paged_token_attention_workspace_bytes(64, 1, 32, 8, 128, 128)
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    _attn(batch=63, hq=32, hkv=8, dh=128, stride=128, ws_bytes=need)
    assert b"too small" not in N.load().last_error()


@pytest.mark.parametrize("call", [
    # one token for each of 2^20 sequences, 16 KV heads: 33 work groups a row
    lambda: _append(rows=1 << 20, seqs=1 << 20, hq=16, hkv=16, qs=1024, ks=1024, vs=1024),
    lambda: _append(rows=1 << 24, seqs=1, hq=2, qs=128, ks=128, vs=128),
    lambda: _select(batch=1 << 20, hq=16, hkv=16),
    lambda: _select(batch=1 << 20, hq=4, hkv=4, stride=8000),
])
def test_more_work_groups_than_a_launch_takes(call):
    assert call() == N.INVALID_ARG
    assert b"for one call" in N.load().last_error()


@pytest.mark.parametrize("device", ["cpu", "meta"])
def test_rope_table_is_made_on_a_gpu(device):
    with pytest.raises(PdecError, match="GPU"):
        paged.rope_table(8, 64, device=device)


@pytest.mark.parametrize("max_pos", [1 << 31, (1 << 32) + 8])
def test_rope_table_refuses_more_positions_than_its_type_counts(max_pos):
    with pytest.raises(PdecError, match="table size"):
        paged.rope_table(max_pos, 2)
