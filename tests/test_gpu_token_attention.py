"""paged_token_attention against the float64 oracle.

Tolerance of an output element, with A the same mix of |v| in the place of v:
  2^-8 A      the weights' rounding to bf16 before the second product,
  2^-8 |out|  the output's rounding to bf16,
  E A         the scores' fp32 errors in the exponent, E = 2 * 2^-24 * (Dh + 4) * max over
              keys of sum_d |q_d k_d| / sqrt(Dh) (both the element's weight and the sum), and
  2^-24 (N + 64) A   sums of N keys in fp32.
"""

import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import operators as oo
from oracle.fp8 import e4m3_decode

pytestmark = pytest.mark.gpu


def _P():
    import paper_2609_36899_amd as P
    return P


class Case:
    """Random pages of which the slots behind each length hold NaN."""

    def __init__(self, lens, hq, hkv, dh, n_q=1, fp8=True, seed=0, share=False):
        rng = np.random.default_rng(seed)
        self.lens = np.asarray(lens, np.int32)
        self.fp8, self.n_q = fp8, n_q
        B = len(lens)
        n = [-(-max(int(x), 0) // 16) for x in lens]
        self.P = sum(n) + 1
        perm = rng.permutation(self.P)
        self.table = rng.integers(0, self.P, (B, max(n + [1]) + 2)).astype(np.int32)
        at = 0
        for b in range(B):
            self.table[b, :n[b]] = perm[at:at + n[b]]
            at += n[b]
        ks, vs = (self.P, hkv, 16, dh), (self.P, hkv, dh, 16)
        if fp8:
            draw = lambda s: (rng.integers(0, 127, s) | (rng.integers(0, 2, s) << 7)).astype(np.uint8)
            self.k, self.v = draw(ks), draw(vs)
            # Scales that are no powers of two, as other writers choose them.
            self.ks = (rng.uniform(0.5, 2.0, (self.P, hkv)) / 200).astype(np.float32)
            self.vs = np.exp2(rng.uniform(-12, 3, (self.P, hkv))).astype(np.float32)
            nan = 0x7F
        else:
            bf = lambda x: torch.from_numpy(x.astype(np.float32)).to(torch.bfloat16).float().numpy()
            self.k, self.v = bf(rng.standard_normal(ks)), bf(rng.standard_normal(vs))
            self.ks = self.vs = None
            nan = np.nan
        for b in range(B):
            if n[b] and lens[b] % 16:
                self.k[self.table[b, n[b] - 1], :, lens[b] % 16:] = nan
                self.v[self.table[b, n[b] - 1], :, :, lens[b] % 16:] = nan
        self.q = torch.from_numpy(rng.standard_normal((B, n_q, hq, dh)).astype(np.float32)
                                  ).to(torch.bfloat16)
        self.selected = None

    def device(self):
        g = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
        k, v = g(self.k), g(self.v)
        if not self.fp8:
            k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        return dict(q=self.q.cuda(), k_pages=k, v_pages=v, block_table=g(self.table),
                    lens=g(self.lens), k_scales=g(self.ks), v_scales=g(self.vs),
                    selected=g(self.selected))

    def run(self):
        d = self.device()
        out = torch.full(d["q"].shape, 9.0, dtype=torch.bfloat16, device="cuda")
        _P().paged_token_attention(out=out, **d)
        torch.cuda.synchronize()
        return out.float().cpu().numpy()

    def values(self):
        if not self.fp8:
            return self.k.astype(np.float64), self.v.astype(np.float64)
        return (e4m3_decode(self.k) * self.ks[:, :, None, None].astype(np.float64),
                e4m3_decode(self.v) * self.vs[:, :, None, None].astype(np.float64))

    def bound(self, ref, size, k):
        q = self.q.float().numpy().astype(np.float64)
        dh = q.shape[-1]
        top = np.abs(np.nan_to_num(k, posinf=0, neginf=0)).max() if k.size else 0.0
        e = 2.0 ** -23 * (dh + 4) * (np.abs(q).sum(-1) * top / np.sqrt(dh))[..., None]
        return (2.0 ** -8 + e + 2.0 ** -24 * (int(self.lens.max()) + 64)) * size + \
            2.0 ** -8 * np.abs(ref) + 1e-30

    def check(self):
        k, v = self.values()
        ref, size = oo.token_attention(self.q.float().numpy(), k, v, self.table, self.lens,
                                       self.selected)
        got = self.run()
        assert np.isfinite(got).all()
        assert (np.abs(got - ref) <= self.bound(ref, size, k)).all(), \
            np.max(np.abs(got - ref) / self.bound(ref, size, k))


EDGE_LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 127, 128, 129, 300, 1000, 2049]
HEADS = [(32, 8, 128), (8, 2, 64), (10, 2, 128), (16, 1, 64), (3, 3, 128), (13, 1, 128)]


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_edge_lengths(hq, hkv, dh, fp8):
    """A long sequence in the batch (its table takes equal stretches), and short ones alone
    (a work group for each)."""
    Case(EDGE_LENS, hq, hkv, dh, fp8=fp8, seed=1).check()
    Case(EDGE_LENS[:-2], hq, hkv, dh, fp8=fp8, seed=1).check()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_q", [2, 3, 4, 5, 8, 9, 17, 40])
def test_several_tokens(n_q, fp8):
    """Lengths below n_q leave tokens without a key: zeros."""
    lens = [0, 1, n_q - 1, n_q, 16, 31, 33, 200, 511]
    Case(lens, 8, 2, 128, n_q=n_q, fp8=fp8, seed=2).check()
    Case(lens + [1500], 8, 2, 128, n_q=n_q, fp8=fp8, seed=2).check()


@pytest.mark.parametrize("hq,hkv,dh,n_q", [(16, 1, 64, 3), (5, 1, 128, 7), (6, 6, 64, 33),
                                            (40, 8, 128, 4), (12, 1, 64, 70), (2, 1, 128, 150)])
def test_several_tokens_of_other_groups(hq, hkv, dh, n_q):
    Case([n_q, 77, 260, 5], hq, hkv, dh, n_q=n_q, seed=3).check()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_q,dh", [(9, 128), (16, 64), (17, 64), (32, 128), (33, 128)])
def test_blocks_of_many_rows(n_q, dh, fp8):
    """36 to 132 rows for a KV head: lengths around two pairs of pages, pages that the table
    does not name, and keys behind some tokens that hold NaN and infinities."""
    lens = [n_q, 63, 64, 65, 95, 96, 97, 128, 129, 161, 700, 2049]
    c = Case(lens, 8, 2, dh, n_q=n_q, fp8=fp8, seed=19)
    c.table[4, 1], c.table[8, 0], c.table[10, 20], c.table[11, 64] = -1, c.P, -5, 2 ** 31 - 1
    c.check()
    for b, n in enumerate(lens):
        page, slot = c.table[b, (n - 1) // 16], (n - 1) % 16
        c.k[page, :, slot] = 0x7F if fp8 else np.nan
        c.v[page, :, :, slot] = 0x7F if fp8 else np.inf
    got = c.run()
    assert np.isnan(got[:, -1]).all()
    k, v = c.values()
    ref, size = oo.token_attention(c.q.float().numpy()[:, :-1], k, v, c.table, c.lens - 1)
    c.q = c.q[:, :-1]
    assert (np.abs(got[:, :-1] - ref) <= c.bound(ref, size, k)).all()


def test_long_contexts_split_over_many_groups():
    Case([40000, 3, 0, 900], 8, 2, 128, seed=4).check()
    Case([20000], 8, 2, 128, n_q=5, fp8=False, seed=5).check()


def test_many_short_sequences():
    """A work group for each; and, with a long one among them, more sequences than one
    prefix-sum step of a work group takes."""
    rng = np.random.default_rng(6)
    lens = rng.integers(0, 40, 700)
    Case(lens, 4, 2, 64, seed=6).check()
    lens[[5, 300]] = 3000, 2500
    Case(lens, 4, 2, 64, seed=6).check()


@pytest.mark.parametrize("fp8", [True, False])
def test_masked_infinities(fp8):
    """What a token does not see may hold anything: keys and values of the tokens after
    it are infinite or NaN, and only the tokens that see them turn NaN."""
    c = Case([37, 64, 19], 8, 2, 64, n_q=4, fp8=fp8, seed=7)
    bad = (0x7F, 0x7F) if fp8 else (np.nan, np.inf)
    for b, n in enumerate(c.lens):
        page, slot = c.table[b, (n - 1) // 16], (n - 1) % 16
        c.k[page, :, slot] = bad[0]
        c.v[page, :, :, slot] = bad[1]
    got = c.run()
    assert np.isnan(got[:, 3]).all()
    k, v = c.values()
    ref, size = oo.token_attention(c.q.float().numpy()[:, :3], k, v, c.table, c.lens - 1)
    c.q, c.n_q = c.q[:, :3], 3
    assert (np.abs(got[:, :3] - ref) <= c.bound(ref, size, k)).all()


def test_scores_of_minus_infinity_and_the_lowest_value():
    """Keys whose scores are -inf weigh nothing; a row that has no others gives zeros."""
    c = Case([20, 16], 2, 1, 64, fp8=False, seed=8)
    c.q = torch.ones_like(c.q)
    low = np.float32(torch.finfo(torch.bfloat16).min)
    c.k[c.table[0, 0], 0, :7] = -np.inf
    c.k[c.table[0, 0], 0, 7:12] = low  # 64 of them: -inf in the sum
    c.k[c.table[1, 0], 0] = -np.inf
    got = c.run()
    keep = np.r_[12:20]
    pages = [c.k[c.table[0, i], 0] for i in (0, 1)], [c.v[c.table[0, i], 0].T for i in (0, 1)]
    k, v = (np.concatenate(p)[keep].astype(np.float64) for p in pages)
    ref, size = oo.mix(np.ones(64), k, v)
    assert (np.abs(got[0, 0] - ref) <= 2.0 ** -7 * size + 1e-6).all()
    assert (got[1] == 0).all()


@pytest.mark.parametrize("fp8", [True, False])
def test_page_ids_outside_the_pool_have_no_keys(fp8):
    c = Case([100, 50, 16, 1700], 8, 2, 64, fp8=fp8, seed=9)
    c.table[0, 2], c.table[0, 5], c.table[1, 0], c.table[2, 0] = -1, c.P, 2 ** 31 - 1, -2 ** 31
    c.check()
    assert (c.run()[2] == 0).all()


@pytest.mark.parametrize("n_q", [1, 3])
@pytest.mark.parametrize("garbage", [np.nan, np.inf, -np.inf, -1.0, 0.0])
def test_pages_that_no_sequence_reads_may_hold_anything(garbage, n_q):
    """Page 0 is nobody's: scales and codes of any kind there reach no output, neither where
    a page stands alone at a sequence's end nor where an id names none."""
    for lens in ([1, 16, 33, 100, 47], [1, 16, 33, 100, 47, 2000]):
        c = Case(lens, 8, 2, 64, n_q=n_q, seed=17)
        used = np.concatenate([c.table[b, :-(-n // 16)] for b, n in enumerate(lens)])
        free = int(np.setdiff1d(np.arange(c.P), used)[0])
        order = np.arange(c.P)
        order[[0, free]] = free, 0
        for name in ("k", "v", "ks", "vs"):
            setattr(c, name, getattr(c, name)[order])
        c.table = order[c.table].astype(np.int32)
        c.k[0], c.v[0] = 0x7F, 0x7F
        c.ks[0], c.vs[0] = garbage, garbage
        want = c.run()
        assert np.isfinite(want).all()
        c.table[3, 2], c.table[4, 0] = -1, c.P
        if n_q == 1:
            pages = max(-(-n // 16) for n in lens)
            c.selected = np.tile(np.arange(pages, dtype=np.int32)[::-1].copy(), (len(lens), 2, 1))
            for b, n in enumerate(lens):
                m = -(-n // 16)
                c.selected[b, :, :m] = np.arange(m)[::-1]
        got = c.run()
        k, v = c.values()
        k[0] = v[0] = 0.0
        ref, size = oo.token_attention(c.q.float().numpy(), k, v, c.table, c.lens, c.selected)
        assert (np.abs(got - ref) <= c.bound(ref, size, k)).all()


@pytest.mark.parametrize("garbage", [np.nan, np.inf, -1.0, 0.0])
def test_listed_pages_behind_the_length_have_no_keys(garbage):
    """A list may name pages of the table that lie behind a length: what they hold, scales
    among it, reaches no output."""
    for lens in ([40, 16, 100], [40, 16, 2000]):
        c = Case(lens, 8, 2, 64, seed=18)
        used = np.concatenate([c.table[b, :-(-n // 16)] for b, n in enumerate(lens)])
        free = int(np.setdiff1d(np.arange(c.P), used)[0])
        c.k[free], c.v[free] = 0x7F, 0x7F
        c.ks[free], c.vs[free] = garbage, garbage
        c.table[0, 5] = c.table[1, 6] = free
        c.selected = np.full((3, 2, 4), -1, np.int32)
        c.selected[0, :, :3] = [5, 2, 0]
        c.selected[1, :, 0] = 6
        c.selected[2] = [4, 3, 6, 0]
        got = c.run()
        k, v = c.values()
        k[free] = v[free] = 0.0
        ref, size = oo.token_attention(c.q.float().numpy(), k, v, c.table, c.lens, c.selected)
        assert (got[1] == 0).all() and (ref[1] == 0).all()
        assert (np.abs(got - ref) <= c.bound(ref, size, k)).all()


@pytest.mark.parametrize("n_q", [1, 9])
def test_value_scales_far_apart(n_q):
    """Scales at the ends of what the append writes, in one row's pages."""
    c = Case([400, 33, 2000], 8, 2, 128, n_q=n_q, seed=20)
    rng = np.random.default_rng(20)
    c.vs = np.exp2(rng.choice([-100, -50, 0, 50, 100], c.vs.shape)).astype(np.float32)
    c.ks = np.where(rng.random(c.ks.shape) < 0.2, np.float32(2.0 ** -100), c.ks)
    c.check()


def test_lengths_past_the_table_are_cut_and_negative_ones_empty():
    c = Case([64, 30], 4, 2, 64, seed=10)
    c.table = np.ascontiguousarray(c.table[:, :4])
    c.check()
    want = c.run()
    c.lens = np.array([70000, -5], np.int32)
    got = c.run()
    np.testing.assert_array_equal(got[0], want[0])
    assert (got[1] == 0).all()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_sel", [1, 2, 3, 9, 64])
def test_selected_pages(n_sel, fp8):
    """Lists in any order, shorter than n_selected, with entries that name nothing."""
    rng = np.random.default_rng(11)
    lens = [0, 1, 16, 33, 200, 1000, 37]
    c = Case(lens, 8, 2, 128, fp8=fp8, seed=11)
    c.selected = np.full((len(lens), 2, n_sel), -1, np.int32)
    for b, n in enumerate(lens):
        pages = -(-n // 16)
        for g in range(2):
            m = min(pages, n_sel)
            c.selected[b, g, :m] = rng.permutation(pages)[:m]
            c.selected[b, g, m:] = rng.integers(-1, 2, n_sel - m)  # behind the list: not read
    c.selected[5, 0, 0] = 2 ** 30
    c.check()


def test_all_pages_selected_equals_none_selected():
    c = Case([1, 100, 555, 2000], 8, 2, 128, seed=12)
    want = c.run()
    c.selected = np.tile(np.arange(125, dtype=np.int32), (4, 2, 1))
    np.testing.assert_array_equal(c.run(), want)


def test_same_call_same_bits_and_page_order():
    c = Case([5, 700, 1500, 33], 8, 2, 128, seed=13)
    a = c.run()
    np.testing.assert_array_equal(a, c.run())
    perm = np.random.default_rng(9).permutation(c.P)
    back = np.argsort(perm)
    for name in ("k", "v", "ks", "vs"):
        setattr(c, name, getattr(c, name)[perm])
    c.table = back[c.table].astype(np.int32)
    np.testing.assert_array_equal(a, c.run())


def test_offsets_past_32_bits():
    """Pages at the end of a pool of more than 2^32 elements."""
    hkv, dh, P = 8, 128, 270000
    k = torch.zeros((P, hkv, 16, dh), dtype=torch.uint8, device="cuda")
    v = torch.zeros((P, hkv, dh, 16), dtype=torch.uint8, device="cuda")
    assert k.numel() > 2 ** 32
    scales = torch.ones((P, hkv), dtype=torch.float32, device="cuda")
    small = Case([40, 90], 8, 8, 128, seed=14)
    d = small.device()
    at = torch.arange(P - small.P, P, device="cuda")
    k[at], v[at] = d["k_pages"], d["v_pages"]
    ks, vs = scales.clone(), scales.clone()
    ks[at], vs[at] = d["k_scales"], d["v_scales"]
    out = torch.empty(d["q"].shape, dtype=torch.bfloat16, device="cuda")
    _P().paged_token_attention(d["q"], k, v, d["block_table"] + (P - small.P), d["lens"], out,
                               k_scales=ks, v_scales=vs)
    np.testing.assert_array_equal(out.float().cpu().numpy(), small.run())


def test_replayed_graph_follows_the_lengths():
    c = Case([300, 80], 8, 2, 64, n_q=2, seed=15)
    d = c.device()
    d["lens"] = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    out = torch.empty(d["q"].shape, dtype=torch.bfloat16, device="cuda")
    eager = torch.empty_like(out)
    ws = torch.empty(_P().paged_token_attention_workspace_bytes(2, 2, 8, 2, 64, 1 << 20),
                     dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _P().paged_token_attention(out=out, workspace=ws, **d)
    for step in range(12):
        graph.replay()
        _P().paged_token_attention(out=eager, workspace=ws, **d)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), step
        d["lens"] += 7


def test_calls_on_two_streams_with_their_own_workspaces():
    c = Case([2000, 700, 33], 8, 2, 128, seed=16)
    d = c.device()
    want = torch.from_numpy(c.run())
    outs = [torch.empty(d["q"].shape, dtype=torch.bfloat16, device="cuda") for _ in range(8)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        _P().paged_token_attention(out=o, stream=streams[i % 2], **d)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o.float().cpu(), want)


@pytest.mark.parametrize("n_q", [1, 5, 13, 26])
@pytest.mark.parametrize("which", ["k", "v", "both"])
def test_a_scale_of_zero_reads_as_zeros(n_q, which):
    """Pages of zeros whose writer left the scale at 0, among others.  It counts as 2^-100:
    whatever finite codes stand there read as 448 * 2^-100 < 2^-91 at most."""
    c = Case([400, 33, 300, 2000, 16], 8, 2, 128, n_q=n_q, seed=21)
    rng = np.random.default_rng(21)
    none = rng.random(c.ks.shape) < 0.3
    none[c.table[1, :3]], none[c.table[4, 0]] = True, True  # sequences of nothing else
    for s, name in ((c.ks, "k"), (c.vs, "v")):
        if which in (name, "both"):
            s[none] = 0.0
            s[c.table[2, 4]] = -0.0
    for selected in (False, True) if n_q == 1 else (False,):
        if selected:
            c.selected = np.stack([rng.permutation(np.arange(127, dtype=np.int32))[:40]
                                   for _ in range(10)]).reshape(5, 2, 40)
        scales = c.ks, c.vs
        got = c.run()
        c.ks, c.vs = (np.maximum(s, np.float32(2.0 ** -100)) for s in scales)
        k, v = c.values()
        ref, size = oo.token_attention(c.q.float().numpy(), k, v, c.table, c.lens, c.selected)
        assert (np.abs(got - ref) <= c.bound(ref, size, k)).all()
        if which != "k":
            assert np.abs(got[[1, 4]]).max() < 2.0 ** -91
        c.ks, c.vs = scales


def _form(c, stride=None):
    """(row tiles a wave, waves along the rows, a work group a unit) of a case's call."""
    lib = ctypes.CDLL(os.path.join(os.path.dirname(_P().__file__), "libpdec_host.so"))
    B, n_q, hq, dh = c.q.shape
    out = (ctypes.c_int32 * 3)()
    lib.pp_paged_attn_form(int(c.fp8), B, n_q, hq, c.k.shape[1], dh, stride or c.table.shape[1],
                           out)
    return tuple(out)


def _widen(c, stride):
    """A table of more pages than any length reaches, with ids of any kind there."""
    rng = np.random.default_rng(30)
    B, have = c.table.shape
    more = rng.integers(-3, c.P + 3, (B, max(stride - have, 0))).astype(np.int32)
    c.table = np.ascontiguousarray(np.concatenate([c.table, more], 1))


def _take_form(c, tiles, waves):
    """Widen the table until a work group's share is one that this form serves."""
    stride = c.table.shape[1]
    while _form(c, stride)[:2] != (tiles, waves):
        stride += stride // 4 + 1
        assert stride < 1 << 20
    _widen(c, stride)
    assert _form(c)[:2] == (tiles, waves)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("tiles,waves", [(1, 2), (2, 1)])
@pytest.mark.parametrize("hq,hkv,dh,n_q", [(8, 2, 128, 5), (8, 2, 64, 8), (3, 1, 64, 8),
                                            (16, 1, 128, 2), (5, 5, 64, 19), (40, 8, 128, 4)])
def test_both_forms_of_17_to_32_rows(hq, hkv, dh, n_q, tiles, waves, fp8):
    """Lengths below n_q and around a pair of pages, ids outside the pool, and then keys and
    values of the last token that hold NaN and infinities."""
    lens = [0, 1, n_q - 1, n_q, n_q + 1, 31, 32, 33, 63, 64, 65, 97, 300, 1000]
    c = Case(lens, hq, hkv, dh, n_q=n_q, fp8=fp8, seed=22)
    _take_form(c, tiles, waves)
    c.table[6, 1], c.table[10, 0], c.table[12, 7], c.table[13, 60] = -1, c.P, -5, 2 ** 31 - 1
    c.check()
    for b, n in enumerate(lens):
        if n >= n_q and b not in (6, 10):
            page, slot = c.table[b, (n - 1) // 16], (n - 1) % 16
            c.k[page, :, slot] = 0x7F if fp8 else np.nan
            c.v[page, :, :, slot] = 0x7F if fp8 else np.inf
    rows = [b for b, n in enumerate(lens) if n >= n_q and b not in (6, 10)]
    got = c.run()
    assert np.isnan(got[rows, -1]).all()
    k, v = c.values()
    ref, size = oo.token_attention(c.q.float().numpy()[:, :-1], k, v, c.table, c.lens - 1)
    c.q = c.q[:, :-1]
    assert (np.abs(got[:, :-1] - ref) <= c.bound(ref, size, k))[rows].all()


@pytest.mark.parametrize("fp8", [True, False])
def test_two_row_tiles_a_wave_with_a_work_group_a_unit(fp8):
    rng = np.random.default_rng(23)
    c = Case(rng.integers(0, 200, 64), 32, 8, 128, n_q=5, fp8=fp8, seed=23)
    _widen(c, 132)
    assert _form(c) == (2, 1, 1)
    c.check()


def _indicator(c, mod):
    """q = 0 and V 1 in dim (pair of pages) % mod: every key weighs the same, so an output is
    the share of a dim's pairs among the keys that a token sees."""
    c.q = torch.zeros_like(c.q)
    c.v[:] = 0
    if c.fp8:
        c.vs[:] = 1.0
    for b, n in enumerate(c.lens):
        for p in range(-(-int(n) // 16)):
            c.v[c.table[b, p], :, p // 2 % mod] = 0x38 if c.fp8 else 1.0


def _shares(lens, n_q, dh, mod):
    """[B][n_q][dh] of what _indicator's call gives."""
    out = np.zeros((len(lens), n_q, dh))
    for b, n in enumerate(lens):
        for j in range(n_q):
            m = int(n) - n_q + j + 1
            if m > 0:
                out[b, j, :mod] = np.bincount(np.arange(m) // 32 % mod, minlength=mod) / m
    return out


def _check_shares(got, lens, n_q, dh, mod):
    """Weights are 1, sums of them whole: the inverse, one product and the bf16 rounding."""
    want = _shares(lens, n_q, dh, mod)[:, :, None]
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -22) * want).all()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_q,tiles,waves", [(1, 1, 1), (4, 1, 1), (5, 1, 2), (5, 2, 1),
                                              (13, 0, 0), (26, 2, 4)])
@pytest.mark.parametrize("lens", [[12000, 3, 0, 900], [20003], "many"])
def test_every_pair_counts_once_where_stretches_meet(lens, n_q, tiles, waves, fp8):
    """A pair of pages that two work groups' stretches lose or share moves an output by
    dh / pairs of it, 5% and more; the tolerance is 2^-8.  Two ways to spread the pairs over
    the dims, so that a lost pair and a doubled one do not make up for each other in both."""
    if lens == "many":
        lens = np.random.default_rng(24).integers(0, 1500, 40)
        lens[[3, 4, 17]] = 0, 9000, 0
        if not fp8 and (tiles, waves) == (1, 2):
            lens = np.minimum(lens, 1600)  # what this form serves of 40 sequences
    dh, hq, hkv = 128, 8, 2
    for mod in (dh, dh - 3):
        c = Case(lens, hq, hkv, dh, n_q=n_q, fp8=fp8, seed=25)
        if tiles:
            _take_form(c, tiles, waves)
        assert not _form(c)[2]
        _indicator(c, mod)
        _check_shares(c.run(), c.lens, n_q, dh, mod)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_q", [1, 5, 13, 26])
def test_replayed_graph_follows_lengths_that_move_the_stretches(n_q, fp8):
    """A table of 200 pairs, so equal stretches: units that end, empty ones and one that takes
    nearly all, with eager calls of the same on other outputs in between."""
    steps = [[3000, 900, 1, 64], [0, 0, 0, 0], [0, 6400, 0, 31], [6400, 6400, 6400, 6400],
             [1, 0, 33, 5000], [n_q, n_q - 1, 2 * n_q, 0], [129, 128, 127, 4000]]
    c = Case([6400] * 4, 8, 2, 128, n_q=n_q, fp8=fp8, seed=26)
    assert not _form(c)[2]
    _indicator(c, 125)
    d = c.device()
    out, eager = (torch.empty(d["q"].shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(_P().paged_token_attention_workspace_bytes(4, n_q, 8, 2, 128,
                                                                c.table.shape[1]),
                     dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _P().paged_token_attention(out=out, workspace=ws, **d)
    for lens in steps + steps[::-1]:
        d["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        out.fill_(7.0)
        graph.replay()
        _P().paged_token_attention(out=eager, workspace=ws, **d)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16)), lens
        _check_shares(out.float().cpu().numpy(), lens, n_q, 128, 125)


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("hq,hkv,n_q", [(16, 1, 4096), (8, 2, 1030), (3, 1, 2000)])
def test_thousands_of_tokens(hq, hkv, n_q, fp8):
    """Prompts: blocks of 128 rows of a KV head, each with its own end of the keys."""
    c = Case([n_q, n_q + 900, 100, n_q - 1], hq, hkv, 64, n_q=n_q, fp8=fp8, seed=27)
    for mod in (64, 61):
        _indicator(c, mod)
        _check_shares(c.run(), c.lens, n_q, 64, mod)


@pytest.mark.parametrize("fp8", [True, False])
def test_every_listed_page_counts_once(fp8):
    """Lists of hundreds of pages, in any order, cut into equal stretches."""
    lens = [9000, 40, 0, 3001]
    c = Case(lens, 8, 2, 128, fp8=fp8, seed=28)
    _indicator(c, 128)
    rng = np.random.default_rng(28)
    want = np.zeros((4, 1, 2, 128))
    c.selected = np.full((4, 2, 300), -1, np.int32)
    for b, n in enumerate(lens):
        pages = -(-n // 16)
        for g in range(2):
            take = rng.permutation(pages)[:300]
            c.selected[b, g, :len(take)] = take
            for p in take:
                want[b, 0, g, p // 2 % 128] += min(16, n - 16 * p)
    want /= np.maximum(want.sum(-1, keepdims=True), 1)
    got = c.run()
    want = want.repeat(4, axis=2)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -22) * want).all()


@pytest.mark.parametrize("fp8", [True, False])
@pytest.mark.parametrize("n_q", [1, 5, 13, 26])
def test_a_broken_query_breaks_its_row_alone(n_q, fp8):
    c = Case([300, 2500], 8, 2, 128, n_q=n_q, fp8=fp8, seed=29)
    want = c.run()
    c.q[0, n_q // 2, 3, 5] = float("nan")
    c.q[1, n_q - 1, 6, 100] = float("inf")
    got = c.run()
    bad = np.zeros(got.shape[:3], bool)
    bad[0, n_q // 2, 3] = bad[1, n_q - 1, 6] = True
    assert np.isnan(got[bad]).all()
    np.testing.assert_array_equal(got[~bad], want[~bad])
