"""Pins of oracle/beam.py: closed forms, exhaustive enumeration, and the rules of ties, masks and
empty slots, by hand."""
import itertools
import math

import numpy as np
import pytest

from oracle import beam


def test_uniform_rows_and_ties():
    # equal scores: lower beam first, then lower token
    out = beam.beam_step(np.zeros((1, 3, 4)), np.zeros((1, 3), np.float32), 6)
    assert out["parent"][0].tolist() == [0, 0, 0, 0, 1, 1]
    assert out["token"][0].tolist() == [0, 1, 2, 3, 0, 1]
    assert np.allclose(out["score"], -math.log(4), atol=1e-15)


def test_known_distribution_and_temperature():
    p = np.array([0.5, 0.25, 0.25])
    out = beam.beam_step(2.0 * np.log(p)[None, None], np.array([[-1.0]], np.float32), 3, T=2.0)
    assert np.allclose(out["score"][0], -1.0 + np.log(p), atol=1e-15)
    assert out["token"][0].tolist() == [0, 1, 2]


def test_masks_dead_and_empty_rows():
    z = np.array([[[0.0, -np.inf, 1.0], [-np.inf] * 3, [np.nan, 0.0, 0.0], [np.inf, 0.0, 0.0],
                   [5.0, 5.0, 5.0]]])
    sc = np.array([[0.0, 0.0, 0.0, 0.0, -np.inf]], np.float32)
    out = beam.beam_step(z, sc, 4)
    assert out["parent"][0].tolist() == [0, 0, -1, -1]
    assert out["token"][0].tolist() == [2, 0, -1, -1]
    assert out["score"][0, 2] == -np.inf


def test_lowest_finite_masks_count_but_rank_last():
    low = float(np.finfo(np.float32).min)
    out = beam.beam_step(np.array([[[0.0, low, 0.0]]]), np.zeros((1, 1), np.float32), 3)
    assert out["token"][0].tolist() == [0, 2, 1]


def test_finished_beams_continue_once():
    z = np.zeros((1, 2, 3))
    out = beam.beam_step(z, np.array([[-1.0, -2.0]], np.float32), 4, done=np.array([[0, 1]]), eos=2)
    # -1 - log 3 = -2.0986 for three tokens of beam 0, below the finished beam's -2
    assert out["parent"][0].tolist() == [1, 0, 0, 0]
    assert out["token"][0].tolist() == [2, 0, 1, 2]
    assert out["done"][0].tolist() == [1, 0, 0, 1]


def test_beam_search_wide_enough_is_exhaustive():
    # a Markov chain of 3 tokens over 3 steps: with 27 beams the search finds every sequence in order
    rng = np.random.default_rng(5)
    first, z = rng.normal(size=3), rng.normal(size=(3, 3))
    lp = lambda r: r - np.log(np.exp(r).sum())  # noqa: E731
    want = sorted(((lp(first)[a] + lp(z[a])[b] + lp(z[b])[c], (a, b, c))
                   for a, b, c in itertools.product(range(3), repeat=3)), reverse=True)
    hist, score, last = [()], np.zeros((1, 1), np.float64), None
    for step in range(3):
        rows = first[None, None] if step == 0 else z[last][None]
        o = beam.beam_step(rows, score, 27)
        live = o["parent"][0] >= 0
        hist = [hist[p] + (t,) for p, t in zip(o["parent"][0][live], o["token"][0][live])]
        last, score = o["token"][0][live], o["score"][:, live]
    assert hist == [s for _, s in want]
    assert np.allclose(score[0], [s for s, _ in want], atol=1e-12)


def test_reorder_by_hand():
    src = np.arange(12).reshape(1, 3, 4)
    out = beam.beam_reorder(src, src, np.array([[2, 2, -1]]))
    assert out[0].tolist() == [[8, 9, 10, 11], [8, 9, 10, 11], [8, 9, 10, 11]]
    out = beam.beam_reorder(src, src, np.array([[1, 7, 0]]), count=np.array([2]), axis=2)
    assert out[0].tolist() == [[4, 5, 2, 3], [4, 5, 6, 7], [0, 1, 10, 11]]


def test_tree_by_hand():
    #   root: a(-1) b(-2); a: c(-1.5) d(-4); b: e(-2.5)
    score = np.array([[[-1, -2, -np.inf]], [[-1.5, -2.5, -4]]], np.float32)
    parent = np.array([[[0, 0, -1]], [[0, 1, 0]]], np.int32)
    token = np.array([[[10, 11, -1]], [[12, 13, 14]]], np.int32)
    t = beam.draft_tree(score, parent, token, 5)
    assert t["count"].tolist() == [5]
    assert t["token"][0].tolist() == [-1, 10, 11, 12, 13]
    assert t["parent"][0].tolist() == [-1, 0, 0, 1, 2]
    assert t["depth"][0].tolist() == [0, 1, 1, 2, 2]
    assert t["mask"][0].tolist() == [1, 3, 5, 11, 21]
    assert t["cand"][0].tolist() == [[10, 11, -1], [12, -1, -1], [13, -1, -1], [-1] * 3, [-1] * 3]
    t = beam.draft_tree(score, parent, token, 4)  # the best three: a, c, b
    assert t["token"][0].tolist() == [-1, 10, 11, 12]


@pytest.mark.parametrize("seed", range(5))
def test_tree_is_closed_under_parents(seed):
    # scores that rise along a path: a node still ranks no higher than its parent
    rng = np.random.default_rng(seed)
    D, B, K = 4, 3, 6
    score = rng.normal(size=(D, B, K)).astype(np.float32)
    parent = rng.integers(-1, K, size=(D, B, K)).astype(np.int32)
    parent[0] = np.minimum(parent[0], 0)
    t = beam.draft_tree(score, parent, np.zeros((D, B, K), np.int32), 10)
    for b in range(B):
        n = t["count"][b]
        assert all(0 <= t["parent"][b, i] < i for i in range(1, n))
        assert all(t["depth"][b, i] == t["depth"][b, t["parent"][b, i]] + 1 for i in range(1, n))
