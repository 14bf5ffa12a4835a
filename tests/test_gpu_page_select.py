"""paged_select against the float64 oracle: the lists are whole numbers and must be equal.

Scores are sums of exact products in fp64, rounded to fp32 once, on both sides, so they
agree but where a sum lies within 2^-45 or so of a border between two fp32 values."""

import numpy as np
import pytest
import torch

from oracle import operators as oo

pytestmark = pytest.mark.gpu


def _P():
    import paper_2609_36899_amd as P
    return P


def _case(lens, hq, hkv, dh, seed, stride=None):
    rng = np.random.default_rng(seed)
    bf = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16)
    n = [-(-max(int(x), 0) // 16) for x in lens]
    pool = sum(n) + 1
    perm = rng.permutation(pool)
    table = np.zeros((len(lens), stride or max(n + [1]) + 1), np.int32)
    at = 0
    for b, m in enumerate(n):
        table[b, :m] = perm[at:at + m]
        at += m
    q = bf(rng.standard_normal((len(lens), hq, dh)))
    means = bf(rng.standard_normal((pool, hkv, dh)) * np.exp2(rng.standard_normal((pool, 1, 1))))
    return q, means, table, np.asarray(lens, np.int32)


def _run(q, means, table, lens, n_sel, first=1, last=1, **kw):
    B, hkv = q.shape[0], means.shape[1]
    out = torch.full((B, hkv, n_sel), 77, dtype=torch.int32, device="cuda")
    _P().paged_select(q.cuda(), means.cuda(), torch.from_numpy(table).cuda(),
                      torch.from_numpy(lens).cuda(), out, keep_first=first, keep_last=last, **kw)
    torch.cuda.synchronize()
    return out.cpu().numpy()


def _check(q, means, table, lens, n_sel, first=1, last=1):
    want = oo.select_pages(q.float().numpy(), means.float().numpy(), table, lens, n_sel, first, last)
    np.testing.assert_array_equal(_run(q, means, table, lens, n_sel, first, last), want)


@pytest.mark.parametrize("n_sel", [2, 3, 16, 33, 200])
@pytest.mark.parametrize("hq,hkv,dh", [(8, 2, 128), (10, 2, 64), (16, 1, 128), (3, 3, 64),
                                        (32, 8, 128)])
def test_lengths_around_the_selection(n_sel, hq, hkv, dh):
    near = n_sel * 16
    _check(*_case([0, 1, 15, 16, 17, near - 1, near, near + 1, near + 17, 3 * near, 2000], hq, hkv,
                  dh, seed=n_sel), n_sel)


@pytest.mark.parametrize("first,last", [(0, 1), (1, 1), (2, 5), (0, 8), (7, 1), (4, 4)])
def test_kept_pages(first, last):
    _check(*_case([40, 130, 900, 16 * 8, 16 * 9], 8, 2, 64, seed=1), 8, first, last)


@pytest.mark.parametrize("pages", [64, 1024, 1025, 8192, 20000])
def test_long_contexts(pages):
    _check(*_case([16 * pages, 16 * pages - 5], 8, 2, 128, seed=2), 64)


def test_equal_scores_go_to_the_lower_page():
    q, means, table, lens = _case([1000, 2000], 8, 2, 64, seed=3)
    means[:] = means[:1]
    _check(q, means, table, lens, 20)
    q.zero_()
    _check(q, means, table, lens, 20)
    means[::3] *= -1  # -0 and 0 alike
    _check(q, means, table, lens, 20)


def test_infinities_nan_and_bad_pages_count_as_the_extremes():
    q, means, table, lens = _case([700, 700, 700], 8, 2, 64, seed=4)
    means[table[0, 3], 0, 5] = float("nan")
    means[table[0, 9]] = float("inf")   # inf - inf in some heads: NaN, in others +-inf
    means[table[1, 4], :, 1] = torch.finfo(torch.bfloat16).max
    table[2, 6], table[2, 7] = -1, len(means)
    for n_sel in (5, 40, 43):
        _check(q, means, table, lens, n_sel)


def test_a_table_longer_than_the_sequences():
    _check(*_case([300, 20, 0], 4, 2, 128, seed=5, stride=3000), 7)
    q, means, table, lens = _case([300, 20], 4, 2, 128, seed=5)
    _check(q, means, np.ascontiguousarray(table[:, :9]), lens, 5)  # cut lengths


def test_same_bits_twice_and_a_given_workspace():
    c = _case([5000] * 9, 8, 2, 128, seed=6)
    ws = torch.empty(_P().paged_select_workspace_bytes(9, 2, c[2].shape[1]), dtype=torch.uint8,
                     device="cuda")
    a = _run(*c, 50)
    np.testing.assert_array_equal(a, _run(*c, 50, workspace=ws))


def test_replayed_graph_follows_the_lengths():
    q, means, table, lens = _case([3000, 900], 8, 2, 64, seed=7)
    dq, dm, dt = q.cuda(), means.cuda(), torch.from_numpy(table).cuda()
    dl = torch.tensor([10, 1], dtype=torch.int32, device="cuda")
    ws = torch.empty(_P().paged_select_workspace_bytes(2, 2, table.shape[1]), dtype=torch.uint8,
                     device="cuda")
    a, b = (torch.empty((2, 2, 24), dtype=torch.int32, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _P().paged_select(dq, dm, dt, dl, a, workspace=ws)
    for _ in range(10):
        graph.replay()
        _P().paged_select(dq, dm, dt, dl, b, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        dl += 83


@pytest.mark.parametrize("hq,hkv,dh", [(9, 9, 64), (16, 16, 128), (20, 20, 64), (36, 12, 128),
                                        (160, 10, 64)])
def test_more_kv_heads_than_a_work_group_takes(hq, hkv, dh):
    """A page's KV heads by two or three work groups, the last with heads to spare."""
    _check(*_case([0, 33, 1700, 16 * 70, 16 * 129 + 1], hq, hkv, dh, seed=8), 12)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (11, 11)])
@pytest.mark.parametrize("B", [511, 512, 513, 1100])
def test_more_sequences_than_a_work_group_has_threads(B, hq, hkv):
    lens = np.random.default_rng(9).integers(0, 130, B)
    lens[[0, 5, B - 1]] = 0, 4000, 1500
    _check(*_case(lens, hq, hkv, 64, seed=9), 5)


@pytest.mark.parametrize("pages", [300, 4000, 9000])
@pytest.mark.parametrize("spread", ["outlier", "two values", "tiny", "least", "huge"])
def test_ranges_that_one_histogram_does_not_part(pages, spread):
    """A score far above the rest, which then share one bin; many equals; scores at the ends
    of fp32, subnormal ones among them (q of 2^-70 and means of 2^-60 .. 2^-75)."""
    q, means, table, lens = _case([16 * pages], 4, 2, 64, seed=10)
    rng = np.random.default_rng(10)
    if spread == "outlier":
        means[table[0, pages // 2]] *= 2.0 ** 60
        means[table[0, pages // 3]] *= -2.0 ** 60
    elif spread == "two values":
        means[:] = torch.where(torch.from_numpy(rng.random((len(means), 1, 1)) < 0.3), means[:1],
                               means[1:2])
    elif spread in ("tiny", "least"):
        q *= 2.0 ** -70
        means *= 2.0 ** (-60 if spread == "tiny" else -75)
    else:
        q *= 2.0 ** 60
        means *= 2.0 ** 62
    _check(q, means, table, lens, 40)
    _check(q, means, table, lens, pages - 3)


def test_offsets_past_32_bits():
    """Means at the end of a pool of more than 2^32 bytes."""
    hkv, dh, P = 8, 128, 2200000
    q, means, table, lens = _case([700, 1900], 16, hkv, dh, seed=11)
    big = torch.zeros((P, hkv, dh), dtype=torch.bfloat16, device="cuda")
    assert big.numel() > 2 ** 31
    big[P - len(means):] = means.cuda()
    out = torch.empty((2, hkv, 20), dtype=torch.int32, device="cuda")
    _P().paged_select(q.cuda(), big, torch.from_numpy(table + np.int32(P - len(means))).cuda(),
                      torch.from_numpy(lens).cuda(), out)
    np.testing.assert_array_equal(out.cpu().numpy(), _run(q, means, table, lens, 20))


@pytest.mark.parametrize("kw", [dict(keep_first=1 << 32), dict(keep_last=(1 << 32) + 1),
                                dict(keep_first=-(1 << 32)), dict(keep_last=1 - (1 << 32))])
def test_kept_pages_past_the_arguments_type_are_refused(kw):
    """They would wrap round to numbers that fit."""
    from paper_2609_36899_amd import PdecError
    q, means, table, lens = _case([400], 4, 2, 64, seed=12)
    with pytest.raises(PdecError, match="keep_first"):
        _run(q, means, table, lens, 5, first=kw.get("keep_first", 1), last=kw.get("keep_last", 1))
