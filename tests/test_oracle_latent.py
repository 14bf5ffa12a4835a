"""The oracle of the operators over latents, against torch's own arithmetic and against
each other: the absorbed form is the expanded one with its matrices moved."""

import numpy as np
import pytest
import torch

from oracle import latent as ol

RNG = np.random.default_rng


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_keeps_lengths_and_turns_by_differences(interleaved):
    rng = RNG(1)
    x, y = rng.standard_normal(64), rng.standard_normal(64)
    ang = np.outer(np.arange(50), 10000.0 ** (-np.arange(32) / 32))
    cs = np.stack([np.cos(ang), np.sin(ang)], axis=-1)
    turned = lambda v, p: ol.rotate(v, cs[p], interleaved)
    assert np.isclose(np.linalg.norm(turned(x, 17)), np.linalg.norm(x))
    assert np.isclose(turned(x, 30) @ turned(y, 25), turned(x, 12) @ turned(y, 7))
    if interleaved:  # a complex product
        z = torch.view_as_complex(torch.from_numpy(x).reshape(32, 2))
        w = z * torch.polar(torch.ones(32, dtype=torch.float64), torch.from_numpy(ang[9]))
        assert np.allclose(turned(x, 9), torch.view_as_real(w).reshape(64).numpy())


def test_norm_is_torchs():
    rng = RNG(2)
    x, g = rng.standard_normal(256), rng.standard_normal(256)
    want = torch.nn.functional.rms_norm(torch.from_numpy(x), (256,), torch.from_numpy(g), 1e-5)
    assert np.allclose(ol.norm(x, g, 1e-5), want.numpy())
    assert ol.norm(x, None, 1e-5) is x


def test_mix_is_torchs_softmax():
    rng = RNG(3)
    q, k, v = rng.standard_normal((5, 8)), rng.standard_normal((9, 8)), rng.standard_normal((9, 4))
    seen = rng.random((5, 9)) < 0.5
    seen[0] = False
    seen[1:, 3] = True
    out, size = ol.mix(q, k, v, 0.3, seen)
    s = torch.from_numpy((q @ k.T) * 0.3).masked_fill(torch.from_numpy(~seen), -np.inf)
    want = torch.softmax(s[1:], -1) @ torch.from_numpy(v)
    assert np.allclose(out[1:], want.numpy()) and (out[0] == 0).all() and (size >= abs(out)).all()


def test_absorbed_is_expanded():
    """With k = c U and v = c W, q_c = q U^T over latents and out W are the expanded form."""
    rng = RNG(4)
    R, H, D, lens, nq = 32, 3, 16, [23, 7], 2
    U, W = rng.standard_normal((H, R, D)), rng.standard_normal((H, R, D))
    table = np.array([[3, 0], [1, 9]])
    latents, keys = rng.standard_normal((4, 16, R)), rng.standard_normal((4, 16, 64))
    q = rng.standard_normal((2, nq, H, D + 64))
    absorbed = np.concatenate([np.einsum("bjhd,hrd->bjhr", q[..., :D], U), q[..., D:]], axis=-1)
    out, _, _ = ol.attention(absorbed, latents, keys, table, lens, 0.2)
    got = np.einsum("bjhr,hrd->bjhd", out, W)
    c = np.concatenate([latents[table[b, :-(-n // 16)]].reshape(-1, R)[:n] for b, n in enumerate(lens)])
    r = np.concatenate([keys[table[b, :-(-n // 16)]].reshape(-1, 64)[:n] for b, n in enumerate(lens)])
    want, _, _ = ol.prompt(q.reshape(-1, H, D + 64), np.einsum("sr,hrd->shd", c, U), r,
                           np.einsum("sr,hrd->shd", c, W), [0, 2, 4], [0, 23, 30], 0.2)
    assert np.allclose(got.reshape(-1, H, D), want)


def test_rows_without_a_place_are_left_out():
    table = np.array([[0, 7], [2, 1]])
    got = list(ol.rows([18, 40], [-1, 2, 5], table, 32, 4, 5))
    assert got == [(0, 0, 16, None), (1, 0, 17, None)]
