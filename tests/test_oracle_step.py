"""Pins of the decoding step's references (oracle/step.py)."""

import math

import numpy as np
import pytest
import torch

from oracle.step import attend_row, draw_token, rotate


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 16))
    f = np.array([1.0, 0.3, 0.01])
    pos = np.array([0, 1, 7, 1000, 12345])
    y = rotate(x, pos, f, interleaved=interleaved)
    a, b = (x[:, 0:6:2], x[:, 1:6:2]) if interleaved else (x[:, :3], x[:, 3:6])
    z = (a + 1j * b) * np.exp(1j * pos[:, None] * f)
    got = (y[:, 0:6:2] + 1j * y[:, 1:6:2]) if interleaved else (y[:, :3] + 1j * y[:, 3:6])
    assert np.allclose(got, z, rtol=0, atol=1e-12)
    assert np.array_equal(y[:, 6:], x[:, 6:]) and np.array_equal(y[0], x[0])


def test_rotated_products_depend_on_the_distance():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 8))
    f = 10000.0 ** (-np.arange(4) / 4)
    at = [float(rotate(q, [p + 3], f)[0] @ rotate(k, [p], f)[0]) for p in (0, 5, 100)]
    assert np.allclose(at, at[0], atol=1e-12)


def test_norm_has_unit_mean_square():
    x = np.random.default_rng(3).standard_normal((4, 64)) * 7
    y = rotate(x, [0] * 4, [], weight=np.ones(64))
    assert np.allclose((y ** 2).mean(axis=1), 1)


def test_attention_equals_torch():
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn(n, 8, generator=g, dtype=torch.float64) for n in (1, 9, 9))
    out, lse, _, _ = attend_row(q[0].numpy(), k.numpy(), v.numpy(), 0.5)
    a = 0.5 * (q @ k.T)
    assert np.allclose(out, (torch.softmax(a, 1) @ v)[0].numpy())
    assert abs(lse - float(torch.logsumexp(a, 1))) < 1e-12
    assert attend_row(np.ones(8), np.zeros((0, 8)), np.zeros((0, 8)), 1.0)[1] == -math.inf


def test_draws_follow_the_filtered_law():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.25, 0.05]))
    tokens = lambda **kw: [draw_token(x, (i + 0.5) / 1000, **kw)[0] for i in range(1000)]
    share = lambda t: [t.count(i) / 1000 for i in range(5)]
    assert share(tokens()) == [0.1, 0.4, 0.2, 0.25, 0.05]
    assert share(tokens(top_k=2)) == pytest.approx([0, 0.4 / 0.65, 0, 0.25 / 0.65, 0], abs=2e-3)
    assert share(tokens(top_p=0.7)) == pytest.approx([0, 0.4 / 0.85, 0.2 / 0.85, 0.25 / 0.85, 0], abs=2e-3)
    assert share(tokens(min_p=0.55)) == pytest.approx([0, 0.4 / 0.65, 0, 0.25 / 0.65, 0], abs=2e-3)
    assert set(tokens(temperature=0.0)) == {1}
    assert draw_token(np.array([1.0, 1.0, 0.0]), 0.9, temperature=0.0) == (0, 0.0)
    assert draw_token(np.array([-math.inf, math.nan]), 0.9)[0] == -1
    assert draw_token(np.array([math.inf, 3.0, math.inf]), 0.6) == (2, math.log(0.5))
