"""Pins of the oracle's token draw: hand-worked weights, a brute force over all
runs in exact fractions, frequencies over a grid of uniform numbers, and the
degenerate rows."""
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import kap_oracle as O

# weights 8, 4, 2, 1, 1 (sum 16) at indices 2, 0, 4, 1, 3
ROW = np.log(np.array([4.0, 1.0, 8.0, 1.0, 2.0]))


@pytest.mark.parametrize("kw, u, want, prob", [
    (dict(), 0.0, 2, 8 / 16), (dict(), 0.49, 2, 8 / 16), (dict(), 0.51, 0, 4 / 16),
    (dict(), 0.76, 4, 2 / 16), (dict(), 0.9, 1, 1 / 16), (dict(), 0.99, 3, 1 / 16),
    (dict(top_k=2), 0.66, 2, 8 / 12), (dict(top_k=2), 0.67, 0, 4 / 12), (dict(top_k=1), 0.99, 2, 1.0),
    (dict(top_k=4), 0.99, 1, 1 / 15),                    # of two equal logits the first stays
    (dict(top_p=0.49), 0.99, 2, 1.0), (dict(top_p=0.51), 0.99, 0, 4 / 12),
    (dict(top_p=0.76), 0.99, 4, 2 / 14), (dict(top_p=0.0), 0.99, 2, 1.0),
    (dict(top_k=3, top_p=0.84), 0.99, 0, 4 / 12),        # 12 / 14 = 0.857: p of the top-k run
    (dict(top_k=3, top_p=0.87), 0.99, 4, 2 / 14),
    (dict(min_p=0.24), 0.99, 4, 2 / 14), (dict(min_p=0.26), 0.99, 0, 4 / 12),
    (dict(min_p=2.0), 0.99, 2, 1.0), (dict(temperature=0.5), 0.74, 2, 64 / 86),
    (dict(temperature=0.5), 0.75, 0, 16 / 86), (dict(temperature=0.0), 0.9, 2, 1.0),
    (dict(temperature=math.inf), 0.39, 0, 0.2), (dict(temperature=math.inf), 0.99, 3, 0.2),
    (dict(), 1.5, 3, 1 / 16), (dict(), math.nan, 2, 0.5),
])
def test_worked(kw, u, want, prob):
    token, p, _ = O.sample(ROW, u, **kw)
    assert token == want and abs(p - prob) < 1e-12


def test_degenerate_rows():
    inf = math.inf
    assert O.sample([-inf, -inf, math.nan], 0.5)[:2] == (-1, 0.0)
    assert O.sample([-inf, 1.0, -inf], 0.999)[:2] == (1, 1.0)
    assert O.sample([1.0, inf, 2.0, inf], 0.6)[:2] == (3, 0.5)
    assert O.sample([math.nan, 3.0, 3.0], 0.4)[:2] == (1, 0.5)
    assert O.sample([5.0], 0.9, top_k=1, top_p=0.1, min_p=1.0)[:2] == (0, 1.0)
    assert O.sample([-inf, 2.0], 0.99, temperature=inf)[:2] == (1, 1.0)


def test_against_exact_fractions():
    rng = np.random.default_rng(5)
    for _ in range(300):
        n = int(rng.integers(1, 9))
        weights = [int(x) for x in rng.integers(1, 6, n)]
        order = sorted(range(n), key=lambda i: (-weights[i], i))
        k = int(rng.integers(0, n + 2))
        p, q, u = (Fraction(int(rng.integers(1, 100)), 101) for _ in range(3))
        k_run = k if 0 < k < n else n
        runs = [order[:r] for r in range(1, n + 1)]
        w_of = lambda run: sum(weights[i] for i in run)
        p_run = next(r for r in range(1, n + 1) if w_of(runs[r - 1]) >= p * w_of(runs[k_run - 1]))
        q_run = sum(Fraction(w, max(weights)) >= q for w in weights)
        run = runs[min(k_run, p_run, q_run) - 1]
        total, at, want = w_of(run), Fraction(0), None
        for i in run:
            at += weights[i]
            if at > u * total:
                want = i
                break
        got, prob, _ = O.sample(np.log(np.array(weights, float)), float(u), top_k=k, top_p=float(p),
                                min_p=float(q))
        assert got == want and abs(prob - weights[want] / total) < 1e-12


def test_frequencies_over_a_grid():
    rng = np.random.default_rng(6)
    row = rng.standard_normal(20)
    w = np.exp(row / 0.7)
    tokens = [O.sample(row, (i + 0.5) / 4000, temperature=0.7)[0] for i in range(4000)]
    got = np.bincount(tokens, minlength=20) / 4000
    # each token's stretch of the unit interval holds its share of the grid, up to one point
    assert np.all(np.abs(got - w / w.sum()) <= 1.01 / 4000)


def test_distance_to_the_next_outcome():
    # u = 0.49 of weights 8, 4, 2, 1, 1: the boundary at 0.5 is 0.01 away
    assert abs(O.sample(ROW, 0.49)[2] - 0.01) < 1e-12
    assert abs(O.sample(ROW, 0.3, top_p=0.8)[2] - 0.05) < 1e-12      # 0.75 | 0.8: nearer than 0.8 * ...


def test_infinite_logits_at_an_infinite_temperature():
    inf = math.inf
    for kw in (dict(), dict(top_k=3), dict(top_p=0.9), dict(min_p=0.5)):
        assert O.sample([1.0, inf, 2.0, inf], 0.4, temperature=inf, **kw)[:2] == (1, 0.5)
        assert O.sample([1.0, inf, -inf, inf], 0.6, temperature=inf, **kw)[:2] == (3, 0.5)
