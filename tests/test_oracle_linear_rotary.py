"""Pins of the oracle's projection by 4-bit weights and rotary positions: closed forms, invariants, small
cases by hand."""
import math

import numpy as np
import pytest

from oracle import linear_w4, rotary
from oracle.attention import round_bf16


def test_bf16_rounding():
    v = np.float32([1.0, 1 + 2.0 ** -8, 1 + 3 * 2.0 ** -8, -3.0e-41, 5e-41, np.inf])
    assert list(linear_w4.bf16(v)) == [1.0, 1.0, 1 + 2.0 ** -6, 0.0, 2.0 ** -133, np.inf]


def test_quantise_by_hand():
    w = np.zeros((2, 40))
    w[0, :4] = [-1.0, 2.0, 0.5, 0.0]           # range 3, s = 0.2 as bf16
    w[0, 32] = 3.0                             # the second group: lo = 0
    q, s, z = linear_w4.quantise(w, 32)
    assert s[0, 0] == round_bf16(np.float64(0.2)) and z[0, 0] == 5
    assert list(q[0, :4]) == [0, 15, round(0.5 / s[0, 0]) + 5, 5]
    assert z[0, 1] == 0 and q[0, 32] == 15 and (q[0, 33:] == 0).all()
    assert (s[1] == 0).all() and (z[1] == 0).all() and (q[1] == 0).all()
    assert s.shape == (2, 4) and (s[0, 2:] == 0).all()       # groups of the padded row


@pytest.mark.parametrize("group", [32, 64, 128])
def test_quantised_weights_are_near(group):
    w = round_bf16(np.random.default_rng(1).standard_normal((5, 200)))
    q, s, z = linear_w4.quantise(w, group)
    g = np.arange(200) // group
    # half a step of the code, and what the scale's own rounding (2^-9 at most of 15 steps) clips
    assert (np.abs(s[:, g] * (q - z[:, g]) - w) <= s[:, g] * (0.5 + 0.5 + 15 * 2.0 ** -8)).all()
    assert q.min() >= 0 and q.max() <= 15


@pytest.mark.parametrize("K,group", [(8, 32), (128, 128), (136, 64), (320, 32)])
def test_pack_and_unpack(K, group):
    rng = np.random.default_rng(K)
    q = rng.integers(0, 16, (3, K))
    groups = linear_w4.padded(K) // group
    s, z = round_bf16(rng.standard_normal((3, groups))), round_bf16(rng.random((3, groups)) * 15)
    data = linear_w4.pack(q, s, z)
    assert len(data) == 3 * (linear_w4.padded(K) // 2 + 4 * groups)
    for a, b in zip(linear_w4.unpack(data, 3, K, group), (q, s, z)):
        assert np.array_equal(a, b)


def test_places_of_codes():
    q = np.zeros((1, 256), int)
    q[0, 128 + 32 * 2 + 8 * 3 + 5] = 9          # second block, j = 2, a = 3, e = 5: word 14, bits 8 + 16
    data = linear_w4.pack(q, np.zeros((1, 2)), np.zeros((1, 2)))
    word = data[64 + 4 * 14:64 + 4 * 15].view(np.uint32)[0]
    assert word == 9 << 24 and data[:128].astype(int).sum() == 9


def test_apply_is_the_product_of_the_values():
    rng = np.random.default_rng(3)
    q, s, z = rng.integers(0, 16, (4, 96)), rng.random((4, 4)), rng.random((4, 4)) * 15
    x = rng.standard_normal((2, 96))
    y, size = linear_w4.apply(x, q, s, z, 32, bias=np.arange(4.0), residual=np.ones((2, 4)))
    want = sum(x[1, k] * s[2, k // 32] * (q[2, k] - z[2, k // 32]) for k in range(96)) + 2 + 1
    assert y[1, 2] == pytest.approx(want, rel=1e-12) and (size >= np.abs(y)).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_turning_keeps_lengths_and_relative_positions(layout):
    rng = np.random.default_rng(4)
    f = rotary.frequencies(32, 10000.0, "plain")
    q, k = rng.standard_normal((2, 1, 1, 48))
    dots = []
    for p in (0, 5, 100000):
        a, _ = rotary.turn(q, [p + 7], f, 1.0, layout)
        b, _ = rotary.turn(k, [p], f, 1.0, layout)
        dots.append((a * b).sum())
        assert np.linalg.norm(a) == pytest.approx(np.linalg.norm(q), rel=1e-12)
        assert np.array_equal(a[..., 32:], q[..., 32:])
    assert dots[1] == pytest.approx(dots[0], rel=1e-9) and dots[2] == pytest.approx(dots[0], rel=1e-9)
    back, _ = rotary.turn(rotary.turn(q, [77], f, 1.0, layout)[0], [77], -f, 1.0, layout)
    assert np.allclose(back, q, atol=1e-14)


def test_turn_by_hand():
    x = np.arange(1.0, 17.0).reshape(1, 1, 16)
    f = np.full(8, math.pi / 2)
    y, size = rotary.turn(x, [1], f, 2.0, "half")          # (a, b) -> 2 (-b, a)
    assert np.allclose(y[0, 0, :8], -2 * x[0, 0, 8:]) and np.allclose(y[0, 0, 8:], 2 * x[0, 0, :8])
    y, _ = rotary.turn(x, [2], f, 1.0, "interleaved")
    assert np.allclose(y, -x) and size[0, 0, 0] == 2 * (1 + 9)


def test_scaled_frequencies():
    f = rotary.frequencies(64, 10000.0, "plain")
    assert f[0] == 1 and f[-1] == pytest.approx(10000.0 ** (-62 / 64))
    assert np.allclose(rotary.frequencies(64, 10000.0, "linear", 4.0), f / 4)
    b = rotary.frequencies(64, 10000.0, "base", 4.0)
    assert b[0] == 1 and b[-1] == pytest.approx(f[-1] / 4)
    for scaling in ("turns", "index"):
        r = rotary.frequencies(64, 10000.0, scaling, 8.0, 4096.0, 1.0, 32.0)
        turns = 4096 * f / (2 * math.pi)
        assert np.allclose(r[turns > 50], f[turns > 50]) and np.allclose(r[turns < 0.7], f[turns < 0.7] / 8)
        assert (np.diff(r) < 0).all() and (r <= f).all() and (r >= f / 8 * (1 - 1e-12)).all()
