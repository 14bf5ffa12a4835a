"""Pins of the oracle's operators: closed forms and small cases worked out by hand."""

import numpy as np

from oracle import operators as oo
from oracle.fp8 import e4m3_decode


def test_rotation_by_a_quarter_turn_and_its_length():
    x = np.arange(8.0)[None]
    cs = np.array([[0.0, 1.0]] * 4)
    np.testing.assert_array_equal(oo.rotate(x, cs)[0], np.concatenate([-x[0, 4:], x[0, :4]]))
    a = np.random.default_rng(0).uniform(0, 6, 4)
    y = oo.rotate(x, np.stack([np.cos(a), np.sin(a)], 1))
    np.testing.assert_allclose(np.linalg.norm(y), np.linalg.norm(x), rtol=1e-14)


def test_page_scale():
    assert oo.page_scale(448.0) == 1.0 and oo.page_scale(448.1) == 2.0
    assert oo.page_scale(224.0) == 0.5 and oo.page_scale(1.0) == 2.0 ** -8
    assert oo.page_scale(0.0) == 2.0 ** -100 and oo.page_scale(1e38) == 2.0 ** 100


def test_append_scales_and_rounds_earlier_codes_again():
    """A page with the value 1.125 (scale 1) gets a token of 896: scale 2, and 0.5625
    stays exact; a token of 448 * 2^7 takes it to the subnormals, 1.125 / 128 = 4.5 / 512,
    a tie that goes to 4."""
    kp, vp = np.zeros((1, 1, 16, 2), np.uint8), np.zeros((1, 1, 2, 16), np.uint8)
    one, cs = np.ones((1, 1), np.float32), np.tile([1.0, 0.0], (16, 1, 1))
    kp[0, 0, 0] = oo.e4m3_encode(1.125)
    for big, want in ((896.0, 1.125), (448.0 * 128, 4 / 512 * 128)):
        x = np.full((1, 1, 2), big)
        k, v, ks, vs, means, _ = oo.append_rows(x, x, [2], [0, 1], [[0]], cs, 16, kp, vp, one, one)
        assert e4m3_decode(k[0, 0, 0, 0]) * ks[0, 0] == want
        assert e4m3_decode(k[0, 0, 1, 0]) * ks[0, 0] == big
        assert means[0, 0][0] == (want + big) / 2


def test_attention_limits():
    """One key: its value.  Equal keys: the mean of the values a token sees."""
    rng = np.random.default_rng(1)
    v = rng.standard_normal((2, 1, 4, 16))
    k = np.ones((2, 1, 16, 4))
    q = rng.standard_normal((1, 3, 2, 4))
    out, _ = oo.token_attention(q, k, v, np.array([[1, 0]]), [18])
    for j in range(3):
        seen = np.concatenate([v[1, 0].T, v[0, 0].T])[:16 + j]
        np.testing.assert_allclose(out[0, j], np.tile(seen.mean(0), (2, 1)), rtol=1e-12)
    out, _ = oo.token_attention(q, k, v, np.array([[1, 0]]), [2])
    assert (out[0, 0] == 0).all()
    np.testing.assert_allclose(out[0, 1], np.tile(v[1, 0, :, 0], (2, 1)))


def test_selection():
    means = np.zeros((4, 1, 2))
    means[:, 0, 0] = [1, 3, 2, 3]
    q, table = np.array([[[1.0, 0.0], [0.0, 1.0]]]), np.arange(4)[None]
    assert oo.select_pages(q, means, table, [64], 2, 0, 1)[0, 0].tolist() == [1, 3]
    assert oo.select_pages(q, means, table, [64], 3, 1, 1)[0, 0].tolist() == [0, 1, 3]
    assert oo.select_pages(q, means, table, [48], 2, 0, 1)[0, 0].tolist() == [1, 2]
    assert oo.select_pages(q, means, table, [16], 3, 1, 1)[0, 0].tolist() == [0, -1, -1]


def test_verification_by_hand():
    """Target (1/2, 1/4, 1/4), drafter (1/4, 1/2, 1/4): token 0 is always accepted, token 1
    with 1/2, and its replacement is always 0 (the only token with more target mass)."""
    t, d = np.log(np.float32([[2, 1, 1]] * 2))[None], np.log(np.float32([[1, 2, 1]]))[None]
    run = lambda x, u0, u1: oo.verify_drafts(t, d, np.array([[x]]), np.float32([[u0, u1]]), 1.0)
    assert run(0, 0.999, 0.3)[0].tolist() == [[0, 0]]
    assert run(1, 0.49, 0.8)[0].tolist() == [[1, 2]]
    for u in (0.0, 0.5, 0.999):
        tokens, n = run(1, 0.51, u)
        assert tokens.tolist() == [[0, -1]] and n.tolist() == [0]
    # without a drafter's logits: accepted with p, replaced by another token
    run = lambda x, u0, u1: oo.verify_drafts(t, None, np.array([[x]]), np.float32([[u0, u1]]), 1.0)
    assert run(0, 0.49, 0.6)[0].tolist() == [[0, 1]]
    assert [run(0, 0.51, u)[0][0, 0] for u in (0.0, 0.49, 0.51, 0.99)] == [1, 1, 2, 2]
    assert run(7, 0.0, 0.6)[0].tolist() == [[1, -1]]
