"""The float64 oracle of keys and values in pages and of log probabilities, pinned by other things than itself."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import a2sf_oracle as A
from oracle import layer_oracle as L


@pytest.mark.parametrize("past,new,window,sinks", [(0, 1, 1, 0), (0, 5, 100, 0), (7, 3, 4, 2), (3, 4, 1, 0), (9, 2, 3, 20), (0, 6, 2, 1)])
def test_seen_by_counting(past, new, window, sinks):
    m = L.seen(past, new, window, sinks)
    for i in range(new):
        p = past + i
        newest = set(range(max(0, p + 1 - window), p + 1))
        assert set(np.flatnonzero(m[i])) == newest | set(range(min(sinks, p + 1)))


def test_gather_follows_the_table():
    pages = np.arange(5 * 2 * 4 * 3).reshape(5, 2, 4, 3).astype(float)
    got = L.gather(pages, [3, 0], 6)
    assert got.shape == (2, 6, 3)
    assert (got[:, :4] == pages[3]).all() and (got[:, 4:] == pages[0][:, :2]).all()


def test_attention_without_a_window_is_masked_attention():
    g = np.random.default_rng(3)
    q, k, v = (g.normal(size=(1, 6, 64)) for _ in range(3))
    o, size, reach = L.attend(q[0][:, None], k, v, L.seen(0, 6, 6, 0))
    want = A.attention_output(A.causal_probabilities(q[0], k[0]), v[0])
    s = q[0] @ k[0].T / 8.0
    for i in range(6):
        w = [math.exp(x) for x in s[i, : i + 1]]
        for e in range(64):
            plain = sum(a * b for a, b in zip(w, v[0, : i + 1, e])) / sum(w)
            assert abs(o[i, 0, e] - plain) < 1e-12
            assert abs(plain - want[i, e]) < 1e-12
        assert reach[i, 0, 0] >= np.abs(s[i, : i + 1]).max() - 1e-12
    assert (size >= np.abs(o) - 1e-15).all()


def test_uniform_attention_is_the_mean():
    v = np.arange(2 * 7 * 64).reshape(2, 7, 64).astype(float)
    o, _, _ = L.attend(np.zeros((2, 4, 64)), np.ones((2, 7, 64)), v, L.seen(5, 2, 3, 1))
    for i, at in enumerate(([0, 3, 4, 5], [0, 4, 5, 6])):
        for h in range(4):
            assert np.allclose(o[i, h], v[h // 2][at].mean(0), rtol=1e-14)


def test_log_probs_of_whole_weights():
    # weights 1, 2, 5 of 8: logits are their logarithms
    logp, entropy, order = L.log_probs(np.log([1.0, 5.0, 2.0]))
    assert np.allclose(np.exp(logp), [float(Fraction(w, 8)) for w in (1, 5, 2)], rtol=1e-14)
    assert abs(entropy + sum(p * math.log(p) for p in (1 / 8, 5 / 8, 2 / 8))) < 1e-14
    assert order == [1, 2, 0]
    logp, entropy, order = L.log_probs(np.array([3.0, 3.0, -math.inf, 3.0]))
    assert order == [0, 1, 3, 2] and abs(entropy - math.log(3)) < 1e-14 and logp[2] == -math.inf
    assert math.isnan(L.log_probs(np.array([1.0, math.nan]))[1]) and L.log_probs(np.array([-math.inf, math.nan, 0.0]))[2] == [2, 0, 1]
