"""verify_drafts against the oracle: whole numbers, compared for equality.

Both sides take masses as whole numbers from one fp64 exponential; two exponentials that
differ in the last place move a mass of 2^40 by one at most, which decides nothing but at
a distance of 2^-40 from a border."""

import ctypes
import os

import numpy as np
import pytest
import torch

from oracle import operators as oo

pytestmark = pytest.mark.gpu


def _P():
    import paper_2609_36899_amd as P
    return P


def _case(B, T, V, seed, std=3.0, noise=1.0, drafter=True):
    rng = np.random.default_rng(seed)
    target = (rng.standard_normal((B, T + 1, V)) * std).astype(np.float32)
    d = (target[:, :T] + rng.standard_normal((B, T, V)) * noise).astype(np.float32)
    drafts = (d + rng.gumbel(size=d.shape)).argmax(-1).astype(np.int32)
    u = rng.random((B, T + 1)).astype(np.float32)
    return [target, d if drafter else None, drafts, u]


def _run(target, d, drafts, u, temperature=1.0, **kw):
    B, T = drafts.shape
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    tokens = torch.full((B, T + 1), 55, dtype=torch.int32, device="cuda")
    accepted = torch.full((B,), 55, dtype=torch.int32, device="cuda")
    _P().verify_drafts(dev(target), dev(drafts), dev(u), tokens, accepted,
                       temperature=temperature, draft_logits=dev(d), **kw)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), accepted.cpu().numpy()


def _check(case, temperature=1.0):
    want = oo.verify_drafts(*case, temperature)
    got = _run(*case, temperature)
    np.testing.assert_array_equal(got[1], want[1])
    np.testing.assert_array_equal(got[0], want[0])
    return want


@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("B,T,V", [(1, 1, 1), (2, 3, 2), (7, 1, 63), (5, 4, 1000), (3, 2, 8191),
                                    (3, 2, 8193), (2, 3, 32003), (1, 2, 151936), (40, 7, 300)])
def test_sizes(B, T, V, drafter):
    for t in (0.7, 1.0, 1.9):
        _check(_case(B, T, V, seed=B + T, drafter=drafter), t)


@pytest.mark.parametrize("drafter", [True, False])
def test_every_count_of_accepted_drafts_occurs(drafter):
    case = _case(64, 3, 50, seed=1, std=1.0, noise=0.5, drafter=drafter)
    if not drafter:
        # Certain drafts now and then: a logit far above the others.
        for b in range(64):
            for i in range(b % 4):
                case[0][b, i, case[2][b, i]] = 40.0
    _, n = _check(case)
    assert set(n) == {0, 1, 2, 3}


def test_equal_distributions_accept_everything():
    case = _case(20, 5, 700, seed=2, noise=0.0)
    _, n = _check(case)
    assert (n == 5).all()


@pytest.mark.parametrize("u", [0.0, 1.0, -3.0, 7.0, 0.99999994, float("nan")])
def test_uniforms_at_and_past_their_ends(u):
    for drafter in (True, False):
        case = _case(6, 3, 400, seed=3, drafter=drafter)
        case[3][:] = u
        if np.isnan(u):
            got = _run(*case)
            case[3][:] = 0.0  # NaN is clamped to 0
            want = oo.verify_drafts(*case, 1.0)
            np.testing.assert_array_equal(got[0], want[0])
        else:
            _check(case)


def test_draft_ids_outside_the_vocabulary_end_the_drafts():
    case = _case(6, 4, 300, seed=4, noise=0.0)
    for b, (i, x) in enumerate([(0, -1), (1, 300), (2, -2 ** 31), (3, 2 ** 31 - 1), (0, 5000)]):
        case[2][b, i] = x
    _, n = _check(case)
    assert list(n) == [0, 1, 2, 3, 0, 4]


def test_masked_and_broken_logits():
    case = _case(8, 2, 500, seed=5)
    t, d = case[0], case[1]
    t[0, :, 250:] = -np.inf                     # a masked half
    d[0, :, :100] = -np.inf
    t[1, 0, 7] = np.nan
    d[2, 1, 9] = np.nan
    t[3, 0] = -np.inf                           # rows without mass
    t[4, 2] = -np.inf
    d[5, 0] = -np.inf
    t[6, 1, 3] = np.inf
    t[7, 0] = np.nan
    _check(case)
    _check([t, None, case[2], case[3]])


def test_flat_and_peaked_rows():
    case = _case(10, 3, 40000, seed=6, std=0.0, noise=0.0)
    _check(case)
    case = _case(10, 3, 4000, seed=7, std=100.0, noise=50.0)
    _check(case, 0.01)
    _check(case, 1e30)


def test_the_next_token_is_distributed_as_the_targets():
    """One draft each, many trials: the token that follows the prefix, whether the draft
    or its replacement, has the target's probabilities.  Each count is binomial: within 5
    of its deviations."""
    rng = np.random.default_rng(8)
    n, V = 20000, 6
    z, dz = rng.standard_normal(V), rng.standard_normal(V)
    target = np.broadcast_to(z, (n, 2, V)).astype(np.float32)
    d = np.broadcast_to(dz, (n, 1, V)).astype(np.float32)
    drafts = (dz + rng.gumbel(size=(n, V))).argmax(-1).astype(np.int32)[:, None]
    u = rng.random((n, 2)).astype(np.float32)
    p = np.exp(z) / np.exp(z).sum()
    for logits in (d, None):
        tokens, _ = _run(target, logits, drafts if logits is not None else
                         np.full((n, 1), 2, np.int32), u)
        count = np.bincount(tokens[:, 0], minlength=V)
        assert (np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_same_bits_twice_and_a_given_workspace():
    case = _case(9, 3, 20000, seed=9)
    ws = torch.empty(_P().verify_drafts_workspace_bytes(9, 3, 20000, True), dtype=torch.uint8,
                     device="cuda")
    ws.fill_(255)
    a, b = _run(*case), _run(*case, workspace=ws)
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(a[1], b[1])


def test_replayed_graph():
    case = _case(4, 3, 9000, seed=10)
    dev = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in case]
    outs = [(torch.empty((4, 4), dtype=torch.int32, device="cuda"),
             torch.empty(4, dtype=torch.int32, device="cuda")) for _ in range(2)]
    ws = torch.empty(_P().verify_drafts_workspace_bytes(4, 3, 9000, True), dtype=torch.uint8,
                     device="cuda")
    call = lambda o: _P().verify_drafts(dev[0], dev[2], dev[3], *o, draft_logits=dev[1], workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(outs[0])
    for _ in range(6):
        graph.replay()
        call(outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        dev[3].copy_(torch.rand_like(dev[3]))
        dev[0].mul_(0.9)


def _form(B, T, V, drafter):
    """(tokens of a chunk, of a cut) of a call."""
    lib = ctypes.CDLL(os.path.join(os.path.dirname(_P().__file__), "libpdec_host.so"))
    out = (ctypes.c_int32 * 2)()
    lib.pp_verify_form(B, T, int(drafter), V, out)
    return tuple(out)


@pytest.mark.parametrize("B,T,V,drafter,form", [
    (98, 1, 32003, False, (2048, 2048)), (99, 1, 32003, False, (2048, 8192)),
    (99, 1, 32003, True, (8192, 8192)), (13, 3, 151936, False, (2048, 2048)),
    (14, 3, 151936, False, (8192, 2048)), (9, 3, 151937, True, (8192, 2048)),
    (25, 2, 128257, False, (8192, 8192)), (20, 1, 163841, True, (8192, 8192))])
def test_each_way_of_cutting_rows(B, T, V, drafter, form):
    """Both sides of both borders, vocabularies that end inside a part of a cut, and next
    tokens from the first part to the last."""
    assert _form(B, T, V, drafter) == form
    case = _case(B, T, V, seed=B, drafter=drafter)
    case[3][:, T] = np.linspace(0.0, 1.0 - 2.0 ** -24, B, dtype=np.float32)
    case[3][::3, 0] = 0.0  # the first draft is accepted
    tokens, n = _check(case, 0.9)
    assert {0, 1} <= set(n)
    new = tokens[np.arange(B), n]
    assert new.min() < 512 and new.max() >= V // 2048 * 2048


def _sides(case, b, i, temperature, k):
    """u24 d_x and 2^24 p_x of draft i with u = k / 2^24."""
    target, d, drafts, _ = case
    x = drafts[b, i]
    mass, unit = oo._mass(target[b, i], temperature)
    right = 2.0 ** 24 * (float(mass[x]) * unit)
    if d is None:
        return k * 2.0 ** 50, right
    mass, unit = oo._mass(d[b, i], temperature)
    return k * (float(mass[x]) * unit), right


def _make_close(case, b, i, temperature, step):
    """A draft with target mass below the drafter's, and the uniform whose side lies next to
    the border: step 0 is the last that accepts, 1 the first that refuses."""
    target, d, drafts, u = case
    p, unit = oo._mass(target[b, i], temperature)
    p = p.astype(np.float64) * unit
    if d is None:
        x = int(p.argmax())
        q = 2.0 ** 50
    else:
        q, unit = oo._mass(d[b, i], temperature)
        q = q.astype(np.float64) * unit
        ratio = p / np.maximum(q, 1.0)
        x = int(np.where((ratio < 0.99) & (ratio > 2.0 ** -6), q, 0.0).argmax())
        q = q[x]
    drafts[b, i] = x
    k = int(np.ceil(2.0 ** 24 * p[x] / q)) - 1 + step
    assert 2 ** 16 < k < 2 ** 24
    u[b, i] = np.float32(k * 2.0 ** -24)
    left, right = _sides(case, b, i, temperature, k)
    assert abs(left - right) < 2.0 ** -15 * right and (left < right) == (step <= 0)


@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("B,T,V", [(24, 4, 300), (12, 4, 20000), (99, 1, 32003)])
def test_uniforms_next_to_the_border(B, T, V, drafter):
    """Tests that the rows' approximate sums cannot decide: the exact ones of the two rows
    do.  The first draft, a middle one or the last on either side of its border, and all of
    a sequence's drafts just accepted."""
    case = _case(B, T, V, seed=11, std=2.0, drafter=drafter)
    if not drafter:
        # A lookup's token has most of the mass, so that its border is a usual one.
        np.put_along_axis(case[0][:, :T], case[2][..., None].astype(np.int64),
                          np.log(np.float32(V)) + 2.0, 2)
    case[3][:, :T] = 0.0  # accepted
    want = np.full(B, T)
    for b in range(B):
        kind, places = b % 4, (0, T // 2, T - 1)
        for i in places if kind == 3 else places[kind:kind + 1]:
            step = b // 4 % 2 if kind < 3 else -1
            _make_close(case, b, i, 0.8, step)
            if step == 1:
                want[b] = i
    _, n = _check(case, 0.8)
    # every test before the close one, and after it where that accepts, is accepted
    np.testing.assert_array_equal(n, want)


def test_equal_sides_refuse():
    """p / d is 1/2 exactly (flat over 4 and over 2 tokens): u = 1/2 is the first refused."""
    t = np.full((3, 2, 1000), -np.inf, np.float32)
    d = np.full((3, 1, 1000), -np.inf, np.float32)
    t[:, :, [5, 77, 400, 999]] = 1.25
    d[:, :, [5, 400]] = -3.0
    u = np.float32([[0.5 - 2.0 ** -24, 0.3], [0.5, 0.3], [0.5 + 2.0 ** -24, 0.9]])
    tokens, n = _check([t, d, np.full((3, 1), 400, np.int32), u])
    assert list(n) == [1, 0, 0] and list(tokens[1:, 0]) == [77, 999]


@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("temperature", [1e-31, 1e-38, 1e-44])
def test_temperatures_at_which_every_test_is_a_close_one(temperature, drafter):
    """All mass on a row's maxima: ties share it."""
    rng = np.random.default_rng(12)
    case = _case(16, 3, 700, seed=12, drafter=drafter)
    case[0][:] = rng.integers(0, 3, case[0].shape) * (rng.random(case[0].shape) < 0.05)
    if drafter:
        case[1][:] = np.where(rng.random(case[1].shape) < 0.5, case[0][:, :3], 0.0)
    top = case[0][:, :3].argmax(-1).astype(np.int32)
    case[2][:] = np.where(rng.random(top.shape) < 0.8, top, case[2])
    case[3][::2, :3] *= 0.05
    _, n = _check(case, temperature)
    assert len(set(n)) > 1


@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("T", [255, 256, 257, 600, 1024])
def test_hundreds_of_drafts(T, drafter):
    """More drafts than a work group has threads; sequences that refuse early, late and never."""
    case = _case(4, T, 40, seed=13, noise=0.0, drafter=drafter)
    case[3][:, :T] = 0.0
    if not drafter:
        case[2][:] = case[0][:, :T].argmax(-1)
    for b, i in ((0, 3), (1, T - 1), (2, T // 2 + 100)):
        case[0][b, i, case[2][b, i]] = -np.inf  # refused
    _, n = _check(case)
    assert list(n) == [3, T - 1, T // 2 + 100, T]


def test_the_largest_vocabulary():
    for drafter in (True, False):
        case = _case(2, 1, 1 << 22, seed=14, drafter=drafter)
        case[3][:] = [[0.0, 0.7], [0.99, 1.0]]
        _check(case)
