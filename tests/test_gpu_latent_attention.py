"""paged_latent_attention against the float64 oracle.

Tolerance of an output element o, with A the same mix of |c| in the place of c:
  2^-8 (A + |o|)   the weights' rounding to bf16 before the second product, in it and in
                   the sum that normalises it; 2^-8 A once more where a token's scale is
                   no power of two (weight times scale is rounded again),
  2^-8 |o|         the output's rounding to bf16,
  E (A + |o|)      the weights' fp32 errors: E = 2^-24 (R + 68) max sum |q k| scale, of the
                   scores and their exponents, + 2^-22 of the exponential, + 2^-24 (N + 64),
                   sums of N keys in fp32 (and their pieces' rescaling).
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


def _bf(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16)


class Case:
    """Random pages, of which the slots behind each length hold NaN, and their scales too."""

    def __init__(self, lens, heads, n_q=1, latent=256, fp8=False, pow2=True, seed=0, scale=0.07,
                 q_size=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.fp8, self.R, self.scale = np.asarray(lens, np.int32), fp8, latent, scale
        self.pow2 = pow2
        n = [-(-max(int(x), 0) // 16) for x in lens]
        self.P = sum(n) + 1
        perm = rng.permutation(self.P)
        self.table = rng.integers(0, self.P, (len(n), max(n + [1]) + 2)).astype(np.int32)
        at = 0
        for b, m in enumerate(n):
            self.table[b, :m] = perm[at:at + m]
            at += m
        self.k = _bf(rng.standard_normal((self.P, 16, ROPE)))
        if fp8:
            self.codes = (rng.integers(0, 127, (self.P, 16, latent))
                          | (rng.integers(0, 2, (self.P, 16, latent)) << 7)).astype(np.uint8)
            e = rng.integers(-9, -5, (self.P, 16)).astype(np.float64)
            self.ts = np.exp2(e if pow2 else e + rng.random((self.P, 16))).astype(np.float32)
        else:
            self.c = _bf(rng.standard_normal((self.P, 16, latent)))
        self.q = _bf(rng.standard_normal((len(n), n_q, heads, latent + ROPE)) * q_size)
        for b, m in enumerate(n):
            if m and lens[b] % 16:
                self.spoil(self.table[b, m - 1], lens[b] % 16)

    def spoil(self, page, slot0):
        self.k[page, slot0:] = float("nan")
        if self.fp8:
            self.codes[page, slot0:] = 0x7F
            self.ts[page, slot0:] = np.nan
        else:
            self.c[page, slot0:] = float("nan")

    def pages(self):
        if not self.fp8:
            return torch.cat([self.c, self.k], -1).cuda(), None
        raw = np.concatenate([self.codes, self.k.view(torch.uint8).numpy()], axis=-1)
        return torch.from_numpy(raw).cuda(), torch.from_numpy(self.ts).cuda()

    def values(self):
        if not self.fp8:
            return self.c.double().numpy()
        with np.errstate(invalid="ignore"):
            return e4m3_decode(self.codes).astype(np.float64) * self.ts.astype(np.float64)[..., None]

    def args(self):
        pages, scales = self.pages()
        q = self.q.cuda()
        out = torch.full((*q.shape[:-1], self.R), float("nan"), dtype=torch.bfloat16, device="cuda")
        return dict(q=q, pages=pages, block_table=torch.from_numpy(self.table).cuda(),
                    lens=torch.from_numpy(self.lens).cuda(), out=out, softmax_scale=self.scale,
                    scales=scales)

    def run(self, **kw):
        return _P().paged_latent_attention(**{**self.args(), **kw})

    def expected(self):
        """Oracle outputs and their tolerances."""
        out, size, reach = ol.attention(self.q.double().numpy(), self.values(),
                                        self.k.double().numpy(), self.table, self.lens, self.scale)
        n = np.maximum(self.lens, 0)[:, None, None]
        E = 2.0 ** -24 * (self.R + 68) * reach + 2.0 ** -22 + 2.0 ** -24 * (n + 64)
        both = size + np.abs(out)
        tol = 2.0 ** -8 * (both + np.abs(out)) + E[..., None] * both
        return out, tol + (0.0 if self.pow2 else 2.0 ** -8 * size) + 1e-30

    def check(self, got=None):
        got = (self.run() if got is None else got).double().cpu().numpy()
        want, tol = self.expected()
        assert np.isfinite(got).all()
        worst = np.max(np.abs(got - want) / tol)
        assert worst <= 1.0, worst


LENS = [[1], [0, 5, 1], [16, 33, 64], [15, 17, 31, 32, 63, 65], [130, 1, 300], [700, 0, 2, 260]]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("heads", [1, 16, 20])
def test_one_token(lens, heads, latent, fp8):
    Case(lens, heads, latent=latent, fp8=fp8, seed=heads).check()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads,n_q", [(16, 2), (5, 3), (33, 1), (40, 1), (64, 1), (65, 1), (80, 1),
                                       (128, 1), (17, 7), (32, 4), (130, 1), (128, 2), (9, 33)])
def test_row_counts(heads, n_q, latent, fp8):
    Case([100, 3, 261, 64], heads, n_q, latent=latent, fp8=fp8, seed=heads + n_q).check()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [16, 128])
def test_scales_that_are_no_powers_of_two(heads, fp8):
    Case([77, 300], heads, fp8=True, pow2=False, seed=3).check()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,n_q", [(4, 1), (128, 1), (32, 3)])
def test_sharp_and_wide_scores(heads, n_q, fp8):
    """Queries so large that a row's maximum outgrows what came before many times over."""
    Case([900, 130], heads, n_q, fp8=fp8, seed=7, q_size=30.0).check()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("latent", [256, 512])
@pytest.mark.parametrize("heads,B", [(16, 1), (64, 3), (128, 2)])
def test_every_key_counts_once(heads, B, latent, fp8):
    """Equal weights, and each element of the latent nonzero at one key alone: a key lost or
    taken twice where tiles, pieces or groups meet shows in its element."""
    n = [5003, 2049, 97][:B]
    case = Case(n, heads, latent=latent, fp8=fp8, seed=1)
    case.q.zero_()
    for turn in range(3):
        where = [np.unique(np.linspace(0, m - 1, latent - 8 + turn).astype(int)) for m in n]
        one = 0x38 if fp8 else 1.0  # the code of 1
        (case.codes if fp8 else case.c)[...] = 0
        if fp8:
            case.ts[...] = 1.0
        for b, keys in enumerate(where):
            for d, key in enumerate(keys):
                (case.codes if fp8 else case.c)[case.table[b, key // 16], key % 16, d] = one
        got = case.run().double().cpu().numpy()
        for b, keys in enumerate(where):
            want = np.zeros(latent)
            want[:len(keys)] = float(torch.tensor(1.0 / n[b]).to(torch.bfloat16))
            assert (got[b, 0] == want).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [16, 128])
def test_pages_that_are_not_there_have_no_keys(heads, fp8):
    case = Case([200, 65, 16], heads, fp8=fp8, seed=5)
    case.table[0, 2], case.table[0, 12], case.table[1, 1], case.table[2, 0] = -1, case.P, 1 << 30, -7
    case.check()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,n_q", [(3, 5), (32, 4), (100, 3)])
def test_later_tokens_reach_no_earlier_ones(heads, n_q, fp8, bad):
    """A drafted token whose latent is not finite: the tokens before it do not see it."""
    case = Case([70, 64, 9], heads, n_q, fp8=fp8, seed=9)
    want, tol = case.expected()
    for b, n in enumerate(case.lens):
        p = n - n_q + 2  # the third of them
        page, slot = case.table[b, p // 16], p % 16
        if fp8:
            case.codes[page, slot, ::3] = 0x7F
        else:
            case.c[page, slot, ::3] = bad
    got = case.run().double().cpu().numpy()
    assert (np.abs(got[:, :2] - want[:, :2]) <= tol[:, :2]).all()
    assert not np.isfinite(got[:, 2:, :, ::3]).any()


@pytest.mark.parametrize("fp8", [False, True])
def test_lengths_past_the_table_and_below_zero(fp8):
    case = Case([64, 40, 30], 16, 2, fp8=fp8, seed=11)
    case.table = np.ascontiguousarray(case.table[:, :4])
    case.lens = np.array([1 << 30, -5, 1], np.int32)
    got = case.run().double().cpu().numpy()
    case.lens[0] = 64
    want, tol = case.expected()
    assert (np.abs(got - want) <= tol).all() and (got[1] == 0).all() and (got[2, 0] == 0).all()


@pytest.mark.parametrize("fp8", [False, True])
def test_many_sequences_have_a_group_each(fp8):
    rng = np.random.default_rng(0)
    Case(rng.integers(0, 70, 530).tolist(), 2, fp8=fp8, seed=12).check()


@pytest.mark.parametrize("fp8", [False, True])
def test_a_workspace_of_ones_own_serves_smaller_calls(fp8):
    P = _P()
    big = P.paged_latent_attention_workspace_bytes(P.FP8_E4M3 if fp8 else P.BF16, 9, 4, 128, 256, 60)
    ws = torch.full((big,), 0xFF, dtype=torch.uint8, device="cuda")
    for lens, heads, n_q in [([500, 3, 77], 128, 4), ([300] * 9, 128, 1), ([400], 5, 1)]:
        case = Case(lens, heads, n_q, fp8=fp8, seed=13)
        case.check(case.run(workspace=ws))


def test_three_dims_mean_one_token():
    case = Case([50, 20], 7, seed=14)
    a = case.args()
    a.update(q=a["q"][:, 0], out=a["out"][:, 0])
    case.check(_P().paged_latent_attention(**a)[:, None])


@pytest.mark.parametrize("fp8", [False, True])
def test_captured_calls_follow_lengths(fp8):
    case = Case([800, 257], 32, 2, fp8=fp8, seed=15)
    a = case.args()
    ws = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        _P().paged_latent_attention(**a, workspace=ws)
    for lens in ([800, 257], [33, 250], [799, 2], [0, 64]):
        case.lens[:] = lens
        a["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        # What lies behind the shorter lengths is part of no answer.
        graph.replay()
        torch.cuda.synchronize()
        once = a["out"].clone()
        assert torch.equal(once, _P().paged_latent_attention(**a))
        case.check(once)


def test_a_stream_of_its_own():
    case = Case([700, 33], 128, seed=16)
    a = case.args()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = _P().paged_latent_attention(**a, stream=stream)
    stream.synchronize()
    case.check(out)


def test_same_call_same_bits():
    case = Case([3000, 1200, 77], 128, seed=17)
    first = case.run().clone()
    for _ in range(3):
        assert torch.equal(case.run(), first)
