"""paged_latent_append and paged_latent_rows against the float64 oracle.

Tolerances.  The norm in fp32: the sum of R squares and the root are off by at most
2^-24 (R / 2 + 4) relative, the two products 2^-24 each: N = 2^-24 (R / 2 + 8).  A rotation:
three fp32 roundings of values up to |x| + |y|: 2^-22 (|x| + |y|), the table's entries, fp32
themselves, among the oracle's inputs.  Then the page type's rounding: bf16 2^-8, E4M3 2^-4
of the value or, below its normal numbers, 2^-10 in units of the scale.
"""

import numpy as np
import pytest
import torch

from oracle import latent as ol
from oracle.fp8 import e4m3_decode

pytestmark = pytest.mark.gpu
ROPE = 64


def _P():
    import paper_2609_36899_amd as P
    return P


def _typed(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(dtype)


class Append:
    def __init__(self, ctx, new, R=256, fp8=False, src=torch.bfloat16, heads=5, interleaved=True,
                 normed=True, seed=0):
        rng = np.random.default_rng(seed)
        self.R, self.fp8, self.interleaved, self.eps = R, fp8, interleaved, 1e-5
        self.lens = np.asarray(ctx, np.int32) + np.asarray(new, np.int32)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        n, self.stride = int(self.starts[-1]), int(max(-(-self.lens // 16))) + 1
        self.P = int(sum(-(-self.lens // 16))) + 2
        perm, at = rng.permutation(self.P), 0
        self.table = np.zeros((len(new), self.stride), np.int32)
        for b, m in enumerate(-(-self.lens // 16)):
            self.table[b, :m] = perm[at:at + m]
            at += m
        size = np.exp2(rng.integers(-6, 7, (n, 1)))
        self.x = _typed(rng.standard_normal((n, R + ROPE)) * size, src)
        self.q = _typed(rng.standard_normal((n, heads, ROPE)), src)
        self.gain = (1 + 0.3 * rng.standard_normal(R)).astype(np.float32) if normed else None
        width = R + 2 * ROPE if fp8 else R + ROPE
        if fp8:
            self.before = torch.from_numpy(rng.integers(0, 256, (self.P, 16, width)).astype(np.uint8))
            self.scales = torch.from_numpy(rng.random((self.P, 16)).astype(np.float32))
        else:
            self.before = _typed(rng.standard_normal((self.P, 16, width)), torch.bfloat16)
            self.scales = None

    def run(self, **kw):
        P = _P()
        self.rope = P.rope_table(max(int(self.lens.max()), 1), ROPE)
        self.pages = self.before.cuda()
        self.got_scales = self.scales.cuda() if self.fp8 else None
        self.q_out = torch.full(self.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
        args = dict(x=self.x.cuda(), lens=torch.from_numpy(self.lens).cuda(),
                    row_start=torch.from_numpy(self.starts).cuda(),
                    block_table=torch.from_numpy(self.table).cuda(), rope=self.rope,
                    pages=self.pages, scales=self.got_scales,
                    gain=None if self.gain is None else torch.from_numpy(self.gain).cuda(),
                    eps=self.eps, interleaved=self.interleaved, q=self.q.cuda(), q_out=self.q_out)
        args.update(kw)
        P.paged_latent_append(**args)
        return self

    def check(self, limit=None):
        limit = self.stride * 16 if limit is None else limit
        x, q = self.x.double().numpy(), self.q.double().numpy()
        cs = self.rope.double().cpu().numpy()
        gain = None if self.gain is None else self.gain.astype(np.float64)
        slots, q_rows = ol.append(x, self.lens, self.starts, self.table, cs,
                                  min(limit, len(cs)), self.P, gain, self.eps, self.interleaved,
                                  self.fp8, q)
        got_q = self.q_out.double().cpu().numpy()
        for r in range(len(x)):
            if r not in q_rows:
                assert (got_q[r] == 7.0).all()
                continue
            turn = 2.0 ** -22 * self.partners(q[r])
            assert (np.abs(got_q[r] - q_rows[r]) <= 2.0 ** -8 * np.abs(q_rows[r]) + turn).all()
        pages = self.pages.cpu()
        R = self.R
        touched = torch.zeros(self.P, 16, dtype=torch.bool)
        where = {(int(self.table[b, p // 16]), p % 16): r
                 for r, b, p, page in ol.rows(self.lens, self.starts, self.table, min(limit, len(cs)),
                                              self.P, len(x)) if page is not None}
        assert set(where) == set(slots)
        norm = 2.0 ** -24 * (R / 2 + 8) if gain is not None else 0.0
        for (page, slot), (c, k, scale) in slots.items():
            touched[page, slot] = True
            row = pages[page, slot]
            if self.fp8:
                # A scale next to a border of the norm's rounding may be the next one.
                s = float(self.got_scales[page, slot])
                top = np.max(np.abs(c)) * scale
                near = np.isclose(top / 448.0, 2.0 ** np.round(np.log2(top / 448.0)), rtol=2 * norm)
                assert s == scale or near
                got = e4m3_decode(row[:R].numpy()) * s
                c = c * scale
                tol = 2.0 ** -4 * np.abs(c) + s * 2.0 ** -10 + norm * np.abs(c)
                key = row[R:].view(torch.bfloat16).double().numpy()
            else:
                got, key = row[:R].double().numpy(), row[R:].double().numpy()
                tol = (2.0 ** -8 + norm) * np.abs(c) + 1e-38
            assert (np.abs(got - c) <= tol).all()
            turn = 2.0 ** -22 * self.partners(x[where[page, slot], R:])
            assert (np.abs(key - k) <= 2.0 ** -8 * np.abs(k) + turn).all()
        assert torch.equal(pages[~touched], self.before[~touched])
        if self.fp8:
            assert torch.equal(self.got_scales.cpu()[~touched], self.scales[~touched])

    def partners(self, x):
        a = np.abs(x)
        if self.interleaved:
            pair = a[..., 0::2] + a[..., 1::2]
            return np.repeat(pair, 2, axis=-1)
        pair = a[..., :32] + a[..., 32:]
        return np.concatenate([pair, pair], axis=-1)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("src", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ctx,new", [([0], [1]), ([15, 16, 40], [1, 1, 1]), ([0, 7, 100], [33, 0, 9]),
                                     ([3] * 70, [1, 2] * 35)])
def test_append(ctx, new, src, R, fp8):
    Append(ctx, new, R, fp8, src, seed=len(ctx)).run().check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("normed", [False, True])
@pytest.mark.parametrize("heads", [1, 8, 9, 33])
def test_forms(heads, normed, interleaved):
    Append([5, 0], [20, 3], heads=heads, normed=normed, interleaved=interleaved, seed=heads).run().check()
    Append([5, 0], [20, 3], 512, True, torch.float32, heads, interleaved, normed, seed=9).run().check()


@pytest.mark.parametrize("fp8", [False, True])
def test_slices_of_wider_rows_and_queries_in_place(fp8):
    case = Append([10, 0], [7, 30], fp8=fp8, heads=6, seed=4)
    n = len(case.x)
    wide = torch.randn(n, 1000, dtype=torch.bfloat16, device="cuda")
    wide[:, 333:333 + case.R + ROPE] = case.x.cuda()
    heads = torch.randn(n, 6, 128 + ROPE + 5, dtype=torch.bfloat16, device="cuda")
    heads[..., 129:129 + ROPE] = case.q.cuda()
    before = heads.clone()
    part = heads[..., 129:129 + ROPE]
    case.run(x=wide[:, 333:333 + case.R + ROPE], q=part, q_out=part)
    case.q_out = part
    case.check()
    assert torch.equal(heads[..., :129], before[..., :129])
    assert torch.equal(heads[..., 129 + ROPE:], before[..., 129 + ROPE:])


def test_rows_without_a_place_are_left_out():
    case = Append([3, 250, 8, 20], [5, 9, 4, 6], fp8=True, seed=5)
    case.table[0, 0] = -1                # its queries are rotated all the same
    case.table[2, 0] = case.P
    case.lens[3] = 2                     # more rows than tokens
    case.run().check()
    case = Append([3, 0], [5, 9], seed=6)
    case.starts[:] = [2, 7, 12]          # rows 0, 1, 12, 13 are no one's
    case.run().check()
    case.starts[:] = [-3, 2, 40]         # sequences that begin and end outside the call
    case.lens[:] = [8, 30]
    case.table = np.arange(4, dtype=np.int32).reshape(2, 2)
    case.stride = 2
    case.run().check()


def test_positions_past_the_table_or_the_angles():
    case = Append([30], [40], seed=7)
    case.table = np.ascontiguousarray(case.table[:, :3])
    case.stride = 3
    case.run().check(48)
    case.run(rope=_P().rope_table(40, ROPE)).check(40)


def test_values_that_do_not_fit():
    case = Append([0], [4], fp8=True, normed=False, src=torch.float32, seed=8)
    case.x[0, :3] = torch.tensor([float("nan"), float("inf"), -float("inf")])
    case.x[1, :256] = 0.0
    case.x[2, :256] = 1e-38
    case.run()
    row = lambda t: e4m3_decode(case.pages[int(case.table[0, 0]), t, :256].cpu().numpy())
    scale = case.got_scales[int(case.table[0, 0])].cpu().numpy()
    assert (np.abs(row(0)[:3]) == 448).all() and np.isfinite(row(0)).all() and row(0)[2] == -448
    assert (row(1) == 0).all() and scale[1] == 2.0 ** -100 and scale[2] == 2.0 ** -100
    assert scale[0] == 2.0 ** 100  # of the infinities


def test_offsets_past_32_bits():
    """Pages whose bytes lie further than 2^32 from the pool's start."""
    P, pages = _P(), (1 << 32) // (16 * 576 * 2) + 40
    pool = torch.zeros(pages, 16, 576, dtype=torch.bfloat16, device="cuda")
    table = torch.tensor([[pages - 1, 3]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([20], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 20], dtype=torch.int32, device="cuda")
    x = torch.randn(20, 576, device="cuda").to(torch.bfloat16)
    rope = torch.zeros(32, 32, 2, device="cuda")
    rope[..., 0] = 1.0
    P.paged_latent_append(x, lens, starts, table, rope, pool)
    assert torch.equal(pool[pages - 1], x[:16]) and torch.equal(pool[3, :4], x[16:])
    c = torch.empty(20, 512, dtype=torch.bfloat16, device="cuda")
    k = torch.empty(20, 64, dtype=torch.bfloat16, device="cuda")
    P.paged_latent_rows(pool, lens, starts, table, c, k)
    assert torch.equal(torch.cat([c, k], 1), x)
    q = torch.zeros(1, 3, 576, dtype=torch.bfloat16, device="cuda")
    out = torch.empty(1, 3, 512, dtype=torch.bfloat16, device="cuda")
    P.paged_latent_attention(q, pool, table, lens, out, 0.1)
    mean = x[:, :512].double().mean(0)
    size = x[:, :512].double().abs().mean(0)
    # Equal weights, exact; the sum of 20, the division and the output's rounding.
    assert ((out.double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -19 * size).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("R", [256, 512])
@pytest.mark.parametrize("lens", [[1], [16, 0, 33], [5] * 90, [300, 7, 0, 64]])
def test_rows_read_back(lens, R, fp8):
    rng = np.random.default_rng(len(lens))
    case = Append(np.zeros(len(lens), int), lens, R, fp8, seed=2)
    if fp8:  # powers of two, so that what reads back is a bf16 number
        case.scales = torch.exp2(torch.from_numpy(rng.integers(-9, 9, (case.P, 16))).float())
        codes = case.before[..., :R]
        codes[(codes & 0x7F) == 0x7F] = 0x38
    _rows(case, case.starts)
    # The last tokens of each alone, and rows of no one.
    some = np.asarray([min(n, 6) for n in lens])
    _rows(case, np.concatenate([[3], 3 + np.cumsum(some)]).astype(np.int32), extra=5)
    case.table[0, 0] = -1
    _rows(case, case.starts)


def _rows(case, starts, extra=0):
    n = int(starts[-1]) + extra
    c = torch.full((n, case.R), 5.0, dtype=torch.bfloat16, device="cuda")
    k = torch.full((n, ROPE), 5.0, dtype=torch.bfloat16, device="cuda")
    _P().paged_latent_rows(case.before.cuda(), torch.from_numpy(case.lens).cuda(),
                           torch.from_numpy(starts).cuda(), torch.from_numpy(case.table).cuda(), c, k,
                           scales=case.scales.cuda() if case.fp8 else None)
    c, k = c.cpu(), k.cpu()
    held = np.zeros(n, bool)
    for r, b, pos, page in ol.rows(case.lens, starts, case.table, case.stride * 16, case.P, n):
        if page is None:
            continue
        held[r] = True
        row = case.before[page, pos % 16]
        if case.fp8:
            want = e4m3_decode(row[:case.R].numpy()) * float(case.scales[page, pos % 16])
            assert np.array_equal(c[r].float().numpy(), want.astype(np.float32))
            assert torch.equal(k[r], row[case.R:].view(torch.bfloat16)) or \
                torch.equal(k[r].view(torch.int16), row[case.R:].view(torch.int16))
        else:
            assert torch.equal(c[r], row[:case.R]) and torch.equal(k[r], row[case.R:])
    assert (c[~held] == 5.0).all() and (k[~held] == 5.0).all()


def test_captured_append_follows_lengths():
    case = Append([4, 31], [1, 1], fp8=True, heads=3, seed=11)
    case.run()
    a = dict(x=case.x.cuda(), lens=torch.from_numpy(case.lens).cuda(),
             row_start=torch.from_numpy(case.starts).cuda(),
             block_table=torch.from_numpy(case.table).cuda(), rope=case.rope, pages=case.pages,
             scales=case.got_scales, gain=torch.from_numpy(case.gain).cuda(), eps=case.eps,
             q=case.q.cuda(), q_out=case.q_out)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        _P().paged_latent_append(**a)
    for lens in ([5, 32], [1, 17], [2, 3]):
        case.lens[:] = lens
        a["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        case.pages.copy_(case.before)
        case.got_scales.copy_(case.scales)
        graph.replay()
        torch.cuda.synchronize()
        case.check()
