"""Pins of the sampling oracle: cases that can be worked out by hand."""
import math

import numpy as np

from oracle import sample_oracle as so


def test_weights_and_the_kept_sets_by_hand():
    x = np.log(np.array([0.5, 0.25, 0.125, 0.125]))
    w = so.weights(x, 1.0)
    assert np.allclose(w, [1, 0.5, 0.25, 0.25])
    assert so.kept_set(x, w) == [0, 1, 2, 3]
    assert so.kept_set(x, w, top_k=2) == [0, 1]
    assert so.kept_set(x, w, top_k=3) == [0, 1, 2]                     # the lower index of the tie
    assert so.kept_set(x, w, top_p=0.4) == [0]
    assert so.kept_set(x, w, top_p=0.6) == [0, 1]
    assert so.kept_set(x, w, top_p=0.7, top_k=2) == [0, 1]             # 0.5 / 0.75 < 0.7
    assert so.kept_set(x, w, top_p=0.6, top_k=2) == [0]                # 0.5 / 0.75 >= 0.6
    assert so.kept_set(x, w, min_p=0.3) == [0, 1]
    assert so.kept_set(x, w, top_p=0.0) == [0]


def test_tokens_follow_the_running_sum_in_index_order():
    x = np.log(np.array([0.2, 0.5, 0.3]))
    assert [so.token(x, u) for u in (0.0, 0.19, 0.21, 0.69, 0.71, 0.999, 1.0)] == [0, 0, 1, 1, 2, 2, 2]
    assert [so.token(x, u, top_k=2) for u in (0.0, 0.62, 0.63, 1.0)] == [1, 1, 2, 2]
    assert so.token(x, 0.9, T=0) == 1


def test_degenerate_rows():
    inf = math.inf
    assert so.sample(np.array([[[math.nan, math.nan]]]), np.array([[0.5]])) == 0
    assert so.sample(np.array([[[math.nan, -inf, -inf]]]), np.array([[0.5]])) == 1
    assert so.sample(np.array([[[3.0, inf, 1.0, inf]]]), np.array([[0.6]])) == 3
    assert so.sample(np.array([[[math.nan, -inf, 2.0]]]), np.array([[0.0]])) == 2


def test_frequencies_of_many_draws_are_the_distribution():
    rng = np.random.default_rng(5)
    x = rng.normal(size=6)
    p = np.exp(x) / np.exp(x).sum()
    got = np.bincount([so.token(x, u) for u in rng.random(4000)], minlength=6) / 4000
    assert np.abs(got - p).max() < 5 * math.sqrt(0.25 / 4000)
