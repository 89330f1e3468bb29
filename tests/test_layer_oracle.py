"""The oracle of the operators around the attention, pinned by things other than itself."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import layer_oracle as L


def test_e4m3_values_and_rounding_agree_with_the_format():
    assert L.E4M3[0x7E] == 448.0 and L.E4M3[1] == 2.0 ** -9 and L.E4M3[0x08] == 2.0 ** -6 and math.isnan(L.E4M3[0xFF])
    bits = torch.arange(256, dtype=torch.uint8)
    of_torch = bits.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(L.E4M3, of_torch, equal_nan=True)
    v = np.random.default_rng(1).uniform(-448, 448, 4000) * 2.0 ** np.random.default_rng(2).integers(-18, 1, 4000)
    ours = L.to_e4m3(v)
    of_torch = torch.from_numpy(v).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    near = np.abs(L.E4M3[ours] - v) <= np.abs(L.E4M3[of_torch] - v)
    assert near.all() and (ours == of_torch).mean() > 0.99


@pytest.mark.parametrize("top,byte", [(448.0, 127), (448.1, 128), (224.0, 126), (224.01, 127), (0.0, 0), (1e-45, 0),
                                      (math.inf, 255), (math.nan, 255), (3.0e38, 247)])
def test_scale_byte(top, byte):
    assert L.scale_byte(np.array([0.0, -top, top / 2])) == byte


def test_norm_and_gate_by_hand():
    h, y = L.rms_norm(np.array([[3.0, 1.0]]), np.array([[0.0, 3.0]]), np.array([2.0, 1.0]), 0.0)
    assert h.tolist() == [[3.0, 4.0]]
    assert np.allclose(y, [[6 / math.sqrt(12.5), 4 / math.sqrt(12.5)]])
    assert np.allclose(L.gated(np.array([2.0, 5.0, 1.0]), np.array([0.0, 1.0, -800.0])), [0.0, 5 / (1 + math.exp(-1)), 0.0])


def test_rotation_keeps_lengths_adds_angles_and_turns_back():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 16))
    f = L.frequencies(12, 10000.0)
    assert f[0] == 1.0 and np.allclose(f[1:] / f[:-1], 10000 ** (-1 / 6))
    for neighbours in (False, True):
        turn = lambda v, p, inv=False: L.rotate(v, np.cos(p * f), np.sin(p * f), 12, neighbours, inv)
        assert np.allclose(turn(turn(x, 3), 4), turn(x, 7))
        assert np.allclose(turn(turn(x, 9), 9, True), x)
        # the product of two turned rows goes by the distance of their positions only
        assert np.allclose((turn(x, 11) * turn(x[::-1], 4)).sum(1), (turn(x, 7) * x[::-1]).sum(1))
        assert np.array_equal(turn(x, 5)[:, 12:], x[:, 12:])


def test_scaled_frequencies():
    f, s = L.frequencies(64, 10000.0), L.frequencies(64, 10000.0, 4.0)
    assert np.allclose(s, f / 4)
    s = L.frequencies(64, 10000.0, 4.0, 8192, 1.0, 4.0)
    turns = 8192 * f / (2 * math.pi)
    assert np.allclose(s[turns >= 4], f[turns >= 4]) and np.allclose(s[turns <= 1], f[turns <= 1] / 4)
    assert ((s <= f) & (s >= f / 4)).all()


def test_sampling_filters_by_hand():
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    one = np.ones(4)
    assert L.sample(l, one) == (1, pytest.approx(0.4))
    assert L.sample(l, np.array([1.0, 9.0, 9.0, 1.0])) == (3, pytest.approx(0.3))
    assert L.sample(l, np.array([0.01, 1.0, 1.0, 1.0]), top_k=3) == (1, pytest.approx(0.4 / 0.9))
    assert L.sample(l, np.array([0.01, 9.0, 0.1, 1.0]), top_p=0.6) == (3, pytest.approx(0.3 / 0.7))
    assert L.sample(l, np.array([0.01, 9.0, 0.1, 1.0]), min_p=0.6) == (3, pytest.approx(0.3 / 0.7))
    assert L.sample(l, np.array([0.01, 9.0, 0.1, 1.0]), temperature=0.0) == (1, 1.0)
    assert L.sample(np.array([2.0, 2.0, 2.0]), np.ones(3), top_k=2) == (0, 0.5)
    assert L.sample(np.array([-math.inf, math.nan]), np.ones(2)) == (-1, 0.0)
    assert L.sample(np.array([0.0, math.inf, math.inf]), np.array([1.0, 2.0, 1.0])) == (2, 0.5)


def test_the_race_draws_each_token_with_its_probability():
    rng = np.random.default_rng(4)
    p = [Fraction(1, 10), Fraction(4, 10), Fraction(2, 10), Fraction(3, 10)]
    l = np.log(np.array([float(x) for x in p]))
    count = np.zeros(4)
    for _ in range(8000):
        count[L.sample(l, rng.exponential(size=4))[0]] += 1
    for c, x in zip(count, p):  # five standard deviations
        assert abs(c / 8000 - float(x)) < 5 * math.sqrt(float(x * (1 - x)) / 8000)
