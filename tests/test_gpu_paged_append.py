"""paged_kv_append against the float64 oracle.

Tolerances.  A rotated element is a sum of two products in fp32: off by at most
2 * 2^-24 (|a c| + |b s|) <= 2^-22 |x| over the pair's largest |x|; the page or q_out
rounding adds half a step of the result (2^-8 relative in bf16, 2^-4 in E4M3, or half of
the smallest step 2^-9 times the page's scale).  V is not rotated, so its codes, the codes
that a growing scale rounds again, and every scale are compared for equality, as are
slots, pages and rows that must not change.
"""

import numpy as np
import pytest
import torch

from oracle import operators as oo
from oracle.fp8 import e4m3_decode

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _P():
    import paper_2609_36899_amd as P
    return P


def _bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


class Case:
    """A pool, a table and rows of one call; pages start out as random garbage."""

    def __init__(self, lens, new, hq, hkv, dh, kind, src, seed=0, means=True, pad=0, spread=1.0,
                 row0=0, behind=0):
        rng = np.random.default_rng(seed)
        self.kind, self.src, self.dh, self.hq, self.hkv = kind, src, dh, hq, hkv
        self.lens, self.new = np.asarray(lens, np.int32), np.asarray(new, np.int32)
        B = len(lens)
        n_pages = [-(-int(n) // 16) for n in lens]
        self.P = sum(n_pages) + 2
        perm = rng.permutation(self.P)
        self.table = np.zeros((B, max(n_pages + [1]) + 1), np.int32)
        at = 0
        for b, n in enumerate(n_pages):
            self.table[b, :n] = perm[at:at + n]
            at += n
        self.starts = (row0 + np.concatenate([[0], np.cumsum(self.new)])).astype(np.int32)
        self.N = int(self.starts[-1]) + behind
        rows = rng.standard_normal((self.N, hq + 2 * hkv, dh + pad)) * spread
        rows *= np.exp2(rng.standard_normal((self.N, 1, 1)))
        td = torch.bfloat16 if src == "bf16" else torch.float32
        # Rows of q|k|v, at element alignment where there is padding.
        flat = torch.from_numpy(rows.reshape(self.N, -1).astype(np.float32)).to(td).cuda()
        width = (hq + 2 * hkv) * dh
        self.rows = flat[:, pad:pad + width] if pad else flat
        cut = lambda a, n: self.rows[:, a * dh:(a + n) * dh].unflatten(1, (n, dh))
        self.q, self.k, self.v = cut(0, hq), cut(hq, hkv), cut(hq + hkv, hkv)
        kshape, vshape = (self.P, hkv, 16, dh), (self.P, hkv, dh, 16)
        self.ks = self.vs = self.means = None
        if kind == "fp8":
            # Every finite code; what was written before this call is read back.
            draw = lambda s: (rng.integers(0, 127, s) | (rng.integers(0, 2, s) << 7)).astype(np.uint8)
            self.kp, self.vp = (torch.from_numpy(draw(s)).cuda() for s in (kshape, vshape))
            sc = lambda: torch.from_numpy(np.exp2(rng.integers(-9, -5, (self.P, hkv))).astype(np.float32)).cuda()
            self.ks, self.vs = sc(), sc()
        else:
            pt = torch.bfloat16 if kind == "bf16" else torch.float32
            self.kp = torch.from_numpy(rng.standard_normal(kshape).astype(np.float32)).to(pt).cuda()
            self.vp = torch.from_numpy(rng.standard_normal(vshape).astype(np.float32)).to(pt).cuda()
        if means and kind != "f32":
            self.means = torch.full((self.P, hkv, dh), 7.0, dtype=torch.bfloat16, device="cuda")
        self.max_pos = max(int(self.lens.max()), 1) if B else 1
        self.rope = _P().rope_table(self.max_pos, dh, 10000.0)
        qt = torch.float32 if kind == "f32" else torch.bfloat16
        self.q_out = torch.full((self.N, hq, dh), 3.0, dtype=qt, device="cuda")

    def host(self, t):
        return t.cpu().numpy() if t.dtype in (torch.uint8, torch.float32) else t.float().cpu().numpy()

    def call(self, **kw):
        args = dict(k_scales=self.ks, v_scales=self.vs, k_means=self.means, q=self.q,
                    q_out=self.q_out)
        args.update(kw)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
        _P().paged_kv_append(self.k, self.v, dev(self.lens), dev(self.starts), dev(self.table),
                             self.rope, self.kp, self.vp, **args)
        torch.cuda.synchronize()

    def check(self):
        f64 = lambda t: t.float().cpu().numpy().astype(np.float64)
        before = [self.host(self.kp), self.host(self.vp)]
        scales = [None if s is None else self.host(s) for s in (self.ks, self.vs)]
        limit = min(self.max_pos, self.table.shape[1] * 16)
        rnd = lambda x: _bf16(x).float().numpy().astype(np.float64)
        wide = [a.astype(np.float64) if self.kind != "fp8" else a for a in before]
        ref = oo.append_rows(f64(self.k), f64(self.v), self.lens, self.starts, self.table,
                             f64(self.rope), limit, *wide, *scales,
                             round_page=rnd if self.kind == "bf16" else (lambda x: x), q=f64(self.q))
        rk, rv, rks, rvs, rmeans, rq = ref
        self.call()
        k, v = self.host(self.kp), self.host(self.vp)
        big = 2.0 ** -22 * float(np.abs(f64(self.k)).max(initial=0.0)) * 2
        if self.kind == "fp8":
            np.testing.assert_array_equal(self.host(self.ks), rks)
            np.testing.assert_array_equal(self.host(self.vs), rvs)
            np.testing.assert_array_equal(v, rv)
            # K codes: the oracle's rounding of a value that differs by the rotation's
            # error: one step at most, and only next to a border between two codes.
            dk, dr = e4m3_decode(k), e4m3_decode(rk)
            np.testing.assert_array_equal(np.isnan(dk), np.isnan(dr))
            s = rks[:, :, None, None]
            step = np.maximum(np.abs(dr) * 2.0 ** -3, 2.0 ** -9) * s
            off = np.abs(np.nan_to_num(dk - dr)) * s
            assert (off <= step * 1.0001).all()
            assert (off > 0).mean() <= 1e-3
        else:
            half = EPS[self.kind]
            touched = rk != wide[0]
            assert (np.abs(k - rk) <= half * np.abs(rk) + big).all()
            np.testing.assert_array_equal(k[~touched], before[0][~touched])
            np.testing.assert_array_equal(v, rnd(rv) if self.kind == "bf16" else rv)
        q = self.q_out.float().cpu().numpy()
        qhalf = EPS["f32" if self.kind == "f32" else "bf16"]
        qbig = 2.0 ** -22 * float(np.abs(f64(self.q)).max(initial=0.0)) * 2
        for r in range(self.N):
            if r in rq:
                assert (np.abs(q[r] - rq[r]) <= qhalf * np.abs(rq[r]) + qbig).all()
            else:
                assert (q[r] == 3.0).all()
        if self.means is not None:
            got = self.means.float().cpu().numpy()
            seen = np.zeros(got.shape[:2], bool)
            for (p, g), m in rmeans.items():
                seen[p, g] = True
                # bf16 rounding, the fp32 sum of 16, and a step of one code or two in 16
                # where K codes differ.
                size = 2.0 ** -8 * np.abs(m) + 2.0 ** -20 * (np.abs(m) + big * 2.0 ** 22)
                if self.kind == "fp8":
                    code_off = np.abs(e4m3_decode(k[p, g]) - e4m3_decode(rk[p, g])).sum(0) * rks[p, g]
                    size = size + np.nan_to_num(code_off)
                else:  # a page element on the other side of a rounding border
                    size = size + 2.0 ** -7 * np.abs(rk[p, g]).max() / 16
                assert (np.abs(got[p, g] - m) <= size).all()
            assert (got[~seen] == 7.0).all()


HEADS = [(4, 2, 64), (8, 8, 128), (10, 2, 128), (16, 1, 64), (5, 5, 64)]


@pytest.mark.parametrize("kind,src", [("fp8", "bf16"), ("fp8", "f32"), ("bf16", "bf16"),
                                       ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("hq,hkv,dh", HEADS)
def test_ragged_rows(kind, src, hq, hkv, dh):
    """Single tokens, runs over page borders, sequences without a new token."""
    lens = [1, 16, 17, 40, 33, 0, 70, 5, 100]
    new = [1, 1, 1, 40, 17, 0, 0, 5, 31]
    Case(lens, new, hq, hkv, dh, kind, src, seed=1).check()


@pytest.mark.parametrize("kind,src", [("fp8", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_rows_at_element_alignment_and_beside_the_sequences(kind, src):
    """q|k|v rows cut out of wider ones at an odd offset; rows before the first
    sequence's and behind the last one's are nobody's."""
    Case([20, 3, 64], [7, 3, 50], 6, 3, 64, kind, src, seed=2, pad=3, row0=2, behind=3).check()


def test_decode_batch_and_one_long_prompt():
    rng = np.random.default_rng(5)
    lens = rng.integers(1, 300, 130)
    Case(lens, np.ones(130, int), 8, 2, 128, "fp8", "bf16", seed=3).check()
    Case([1025], [1025], 8, 2, 128, "fp8", "f32", seed=4).check()
    Case([1025], [1020], 8, 2, 128, "bf16", "bf16", seed=4, means=False).check()


@pytest.mark.parametrize("spread", [0.0, 1e-20, 2.0 ** -8, 1e3, 1e30])
def test_scales_of_any_size(spread):
    """Zeros (the smallest scale), tiny and huge keys; part-full pages whose codes move
    to a much larger scale (and vanish) or stay at theirs."""
    Case([9, 30, 47, 16], [3, 30, 1, 4], 4, 2, 64, "fp8", "f32", seed=6, spread=spread).check()


def test_a_scale_that_a_caller_made_is_kept_at_the_next_power_of_two():
    """The page's scale 0.3 becomes 0.5; its codes are rounded again from 0.3."""
    c = Case([9], [1], 2, 2, 64, "fp8", "f32", seed=7, spread=1e-3)
    c.ks.fill_(0.3)
    c.vs.fill_(0.3)
    old = c.kp.cpu().numpy()
    c.call()
    page = c.table[0, 0]
    assert (c.ks[page].cpu().numpy() == 0.5).all()
    want = oo.e4m3_encode(np.float32(e4m3_decode(old[page, :, :8]).astype(np.float32)
                                     * np.float32(0.3)).astype(np.float64) / 0.5)
    np.testing.assert_array_equal(c.kp[page].cpu().numpy()[:, :8], want)


def test_infinities_and_nan_saturate_and_stay_in_their_head():
    c = Case([20], [20], 2, 2, 64, "fp8", "f32", seed=8)
    c.rows[3, c.hq * 64 + 5] = np.inf      # k, head 0, token 3, dim 5 (pair 37)
    c.rows[4, (c.hq + c.hkv) * 64 + 9] = np.nan   # v, head 0, token 4
    c.call()
    page = c.table[0, 0]
    assert float(c.ks[page, 0]) == 2.0 ** 100 and float(c.ks[page, 1]) < 1.0
    assert int(c.kp[page, 0, 3, 5]) & 0x7F == 0x7E
    assert int(c.vp[page, 0, 9, 4]) & 0x7F == 0x7E
    assert float(c.vs[page, 0]) < 1.0


def test_nan_of_any_payload_stays_nan_in_bf16():
    c = Case([4], [4], 2, 2, 64, "bf16", "f32", seed=8)
    c.rows.view(torch.int32)[1] = 0x7FFFFFFF
    c.rows.view(torch.int32)[2] = -1
    c.call()
    page = c.table[0, 0]
    for t in (1, 2):
        assert torch.isnan(c.kp[page, :, t].float()).all()
        assert torch.isnan(c.vp[page, :, :, t].float()).all()
        assert torch.isnan(c.q_out[t].float()).all()
    assert torch.isfinite(c.kp[page, :, 3].float()).all() and torch.isnan(c.means[page].float()).all()


@pytest.mark.parametrize("kind", ["fp8", "bf16"])
def test_what_is_out_of_range_is_left_out(kind):
    """Page ids outside the pool, positions past the angles and past the table, and a
    length smaller than the rows it counts."""
    c = Case([40, 40, 90, 2], [20, 20, 30, 5], 4, 2, 64, kind, "f32", seed=9)
    c.table[0, 1] = c.P
    c.table[1, 2] = -1
    c.max_pos = 80
    c.rope = c.rope[:80].contiguous()
    c.check()
    c = Case([40, 40], [33, 4], 4, 2, 64, kind, "f32", seed=10)
    c.table = np.ascontiguousarray(c.table[:, :2])
    c.check()


def test_lengths_at_the_ends_of_their_type_append_nothing():
    c = Case([40, 40, 40, 40], [4, 4, 4, 4], 4, 2, 64, "fp8", "f32", seed=14)
    before = [t.clone() for t in (c.kp, c.vp, c.ks, c.vs, c.q_out, c.means)]
    c.lens = np.array([-2 ** 31, -2 ** 31 + 2, -1, 2 ** 31 - 1], np.int32)
    c.call()
    for t, old in zip((c.kp, c.vp, c.ks, c.vs, c.q_out, c.means), before):
        assert torch.equal(t, old)


def test_token_by_token_equals_at_once():
    """bf16 pages: the same bytes either way.  E4M3 pages: the same scales, and codes that
    differ only where a growing scale took earlier ones below the normal range."""
    for kind in ("bf16", "fp8"):
        one = Case([50], [50], 4, 2, 128, kind, "f32", seed=11)
        many = Case([50], [50], 4, 2, 128, kind, "f32", seed=11)
        one.call()
        rows = many.rows
        for t in range(50):
            many.lens, many.starts = np.array([t + 1], np.int32), np.array([0, 1], np.int32)
            cut = lambda a, n: rows[t:t + 1, a * 128:(a + n) * 128].unflatten(1, (n, 128))
            many.k, many.v = cut(4, 2), cut(6, 2)
            many.call(q=None, q_out=None)
        pages = one.table[0, :4]
        for a, b in ((one.kp, many.kp), (one.vp, many.vp)):
            a, b = a[pages.tolist()], b[pages.tolist()]
            if kind == "bf16":
                assert torch.equal(a, b)
            else:
                x, y = e4m3_decode(a.cpu().numpy()), e4m3_decode(b.cpu().numpy())
                # stale slots of the last page differ in nothing either
                assert (np.abs(x - y) <= 2.0 ** -9).all()
        if kind == "fp8":
            assert torch.equal(one.ks[pages.tolist()], many.ks[pages.tolist()])
            assert torch.equal(one.vs[pages.tolist()], many.vs[pages.tolist()])


def test_calls_without_rows_or_queries():
    c = Case([5], [5], 4, 2, 64, "bf16", "f32", seed=12)
    before = c.kp.clone()
    c.k, c.v = c.k[:0], c.v[:0]
    c.call(q=None, q_out=None)
    assert torch.equal(before, c.kp)


def test_rope_table_matches_its_definition():
    t = _P().rope_table(5000, 128, 1e6).cpu().numpy().astype(np.float64)
    ang = np.arange(5000)[:, None] * 1e6 ** (-2.0 * np.arange(64) / 128)
    np.testing.assert_allclose(t[..., 0], np.cos(ang), atol=2.0 ** -24 + 1e-11)
    np.testing.assert_allclose(t[..., 1], np.sin(ang), atol=2.0 ** -24 + 1e-11)


def test_replayed_graph_follows_the_lengths():
    """One token a replay, the lengths raised on the device between them, eager work of
    the program's own in between."""
    P = _P()
    c = Case([64, 40], [1, 1], 4, 2, 64, "fp8", "bf16", seed=13)
    eager = Case([64, 40], [1, 1], 4, 2, 64, "fp8", "bf16", seed=13)
    lens = torch.tensor([1, 5], dtype=torch.int32, device="cuda")
    starts, table = torch.from_numpy(c.starts).cuda(), torch.from_numpy(c.table).cuda()
    kw = dict(k_scales=c.ks, v_scales=c.vs, k_means=c.means, q=c.q, q_out=c.q_out)
    ekw = dict(k_scales=eager.ks, v_scales=eager.vs, k_means=eager.means, q=eager.q,
               q_out=eager.q_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.paged_kv_append(c.k, c.v, lens, starts, table, c.rope, c.kp, c.vp, **kw)
    for step in range(36):
        graph.replay()
        P.paged_kv_append(eager.k, eager.v, lens, starts, table, c.rope, eager.kp, eager.vp, **ekw)
        if step % 5 == 0:
            torch.cuda.synchronize()
        for a, b in ((c.kp, eager.kp), (c.vp, eager.vp), (c.ks, eager.ks), (c.vs, eager.vs),
                     (c.means, eager.means), (c.q_out, eager.q_out)):
            assert torch.equal(a, b), step
        lens += 1


@pytest.mark.parametrize("kind", ["fp8", "bf16", "f32"])
@pytest.mark.parametrize("lens,new,first", [([40, 21], [19, 4], -11), ([8, 30], [1, 1], -7),
                                            ([70], [33], -2 ** 31)])
def test_a_sequence_may_begin_before_the_calls_first_row(kind, lens, new, first):
    """Rows of the first sequence that an earlier call appended: row_start[0] below 0 says
    where they would be.  The positions count from the sequence's end, so the call is the
    one with row_start[0] = 0."""
    a, b = (Case(lens, new, 4, 2, 64, kind, "f32", seed=15) for _ in range(2))
    b.starts[0] = first
    a.call()
    b.call()
    for name in ("kp", "vp", "ks", "vs", "means", "q_out"):
        x, y = getattr(a, name), getattr(b, name)
        assert x is None or torch.equal(x, y), name


@pytest.mark.parametrize("kind", ["fp8", "bf16"])
def test_a_sequence_may_end_behind_the_calls_last_row(kind):
    a, b = (Case([40, 29], [19, 14], 4, 2, 64, kind, "f32", seed=16) for _ in range(2))
    b.starts[-1] += 7
    b.lens[-1] += 7
    a.call()
    b.call()
    for name in ("kp", "vp", "ks", "vs", "means", "q_out"):
        x, y = getattr(a, name), getattr(b, name)
        assert x is None or torch.equal(x, y), name


@pytest.mark.parametrize("kind,src", [("fp8", "bf16"), ("bf16", "f32")])
def test_many_uneven_sequences(kind, src):
    """Where a row's sequence lies far from where equal shares would put it."""
    rng = np.random.default_rng(17)
    for big in (0, 299):
        new = rng.integers(0, 4, 300)
        new[big] = 1500
        lens = new + rng.integers(0, 40, 300)
        Case(lens, new, 2, 1, 64, kind, src, seed=17).check()


def test_offsets_past_32_bits():
    """Pages at the end of a pool of more than 2^32 elements."""
    P, hkv, dh = 270000, 8, 128
    a, b = (Case([40, 19], [30, 1], 16, hkv, dh, "fp8", "bf16", seed=18) for _ in range(2))
    a.call()
    at = P - b.P
    small = b.kp, b.vp, b.ks, b.vs, b.means
    big = [torch.zeros((P,) + t.shape[1:], dtype=t.dtype, device="cuda") for t in small]
    assert big[0].numel() > 2 ** 32
    for x, y in zip(big, small):
        x[at:] = y
    b.kp, b.vp, b.ks, b.vs, b.means = big
    b.table = b.table + np.int32(at)
    b.call()
    for x, y in zip(big, (a.kp, a.vp, a.ks, a.vs, a.means)):
        assert torch.equal(x[at:], y)
        assert not x[:at].any()
