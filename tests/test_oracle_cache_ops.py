"""Pins of the cache operators' oracle: hand values, and properties that hold
whatever the implementation (rotation by difference, torch's own attention
probabilities, brute-force selection)."""
import itertools
import math

import numpy as np
import pytest
import torch

import oracle
from oracle.cache_ops import kept_rows


def test_rope_by_hand():
    """Positions 0, 1 and 2 of a head of four with frequencies pi/2 and pi: turns by quarters and halves."""
    x = np.array([[[1.0, 2.0, 3.0, 4.0]]] * 3)
    inv = np.array([math.pi / 2, math.pi])
    half = oracle.rope_rows(x, [0, 1, 2], inv)
    # pairs (1, 3) and (2, 4)
    np.testing.assert_allclose(half[:, 0], [[1, 2, 3, 4], [-3, -2, 1, -4], [-1, 2, -3, 4]], atol=1e-14)
    inter = oracle.rope_rows(x, [0, 1, 2], inv, interleaved=True)
    # pairs (1, 2) and (3, 4)
    np.testing.assert_allclose(inter[:, 0], [[1, 2, 3, 4], [-2, 1, -3, -4], [-1, -2, 3, 4]], atol=1e-14)
    part = oracle.rope_rows(x, [0, 1, 2], inv[:1], magnitude=2.0, interleaved=True)
    np.testing.assert_allclose(part[:, 0], [[2, 4, 3, 4], [-4, 2, 3, 4], [-2, -4, 3, 4]], atol=1e-14)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_products_depend_on_the_difference_of_positions(interleaved):
    g = np.random.default_rng(1)
    q, k = g.standard_normal((1, 2, 16)), g.standard_normal((1, 2, 16))
    inv, _ = oracle.rope_freqs(12)
    dots = [(oracle.rope_rows(q, [m], inv, interleaved=interleaved) * oracle.rope_rows(k, [m - 7], inv, interleaved=interleaved)).sum(-1)
            for m in (0, 7, 123, -5)]
    for d in dots[1:]:
        np.testing.assert_allclose(d, dots[0], atol=1e-12)


def test_rope_frequencies():
    inv, m = oracle.rope_freqs(4, theta=100.0)
    np.testing.assert_allclose(inv, [1.0, 0.1])
    assert m == 1.0
    np.testing.assert_allclose(oracle.rope_freqs(4, 100.0, "linear", 4.0)[0], [0.25, 0.025])
    # theta * s^(4/2): the last pair is slowed by exactly s, the first not at all
    np.testing.assert_allclose(oracle.rope_freqs(4, 100.0, "ntk", 4.0)[0], [1.0, 0.1 / 4.0])
    # 20 pi positions: 10 turns and 1 turn; kept from 10 on, divided from 1 down
    inv, m = oracle.rope_freqs(4, 100.0, "by_parts", 8.0, 20 * math.pi, 1.0, 10.0)
    np.testing.assert_allclose(inv, [1.0, 0.1 / 8.0])
    assert abs(m - (0.1 * math.log(8.0) + 1.0)) < 1e-15
    # halfway between the bounds (5.5 turns for the first pair): the mean of both
    np.testing.assert_allclose(oracle.rope_freqs(2, 100.0, "by_parts", 8.0, 11 * math.pi, 1.0, 10.0)[0], [0.5 + 0.5 / 8.0])


def test_score_is_the_column_sum_of_the_attention_probabilities():
    """Two layers, grouped heads, a path of three tokens after five rows: decay times the old score plus what torch's
    softmax over the causal scores gives each row, summed over tokens and a group's heads."""
    g = np.random.default_rng(3)
    layers, H, Hkv, D, L, n = 2, 4, 2, 8, 5, 6
    path = [0, 2, 5]
    q, k = g.standard_normal((layers, n, H, D)), g.standard_normal((layers, 1, Hkv, 10, D))
    old = g.random((layers, 1, Hkv, 10))
    scale = 0.4
    s = torch.einsum("lihd,lhjd->lhij", torch.tensor(q[:, path]), torch.tensor(k[:, 0]).repeat_interleave(2, 1)) * scale
    mask = torch.arange(10)[None] <= L + torch.arange(3)[:, None]
    s = s.masked_fill(~mask, -math.inf)
    lse = np.zeros((layers, n, H))
    lse[:, path] = torch.logsumexp(s, -1).transpose(1, 2).numpy()
    want = torch.softmax(s, -1).sum(2).view(layers, Hkv, 2, 10).sum(2).numpy()
    want[:, :, :L] += 0.9 * old[:, 0, :, :L]
    want[:, :, 8:] = old[:, 0, :, 8:]
    got, terms = oracle.kv_score(q, lse, k, [L], [0, n], [path], old, scale, 0.9)
    np.testing.assert_allclose(got[:, 0], want, rtol=1e-12)
    # the new weight of all rows: one for each token and head
    np.testing.assert_allclose(terms[0].sum(), layers * 3 * H, rtol=1e-12)


def test_score_of_a_query_that_saw_nothing_is_zero():
    out, _ = oracle.kv_score(np.ones((1, 1, 1, 8)), [[[-np.inf]]], np.ones((1, 1, 1, 4, 8)), [2], [0, 1], [[0]],
                             np.full((1, 1, 1, 4), 7.0), 1.0)
    assert out[0, 0, 0].tolist() == [7.0, 7.0, 0.0, 7.0]


def test_evict_by_hand():
    score = [5.0, 1.0, 3.0, 3.0, 0.0, 9.0, 2.0]
    assert kept_rows(score, 7, 0, 0) == [0, 1, 2, 3, 4, 5, 6]
    assert kept_rows(score, 3, 0, 0) == [0, 2, 5]           # 3.0 twice: the lower row
    assert kept_rows(score, 4, 2, 1) == [0, 1, 5, 6]
    assert kept_rows(score, 2, 1, 1) == [0, 6]              # nothing by score
    assert kept_rows([0.0, -0.0, 0.0, 1.0], 2, 0, 0) == [0, 3]
    assert kept_rows([1.0, math.nan, math.inf, 2.0], 2, 0, 0) == [1, 2]
    assert kept_rows([], 4, 0, 0) == []


def test_evict_keeps_the_most_score():
    """Against every subset of eight rows: no admissible choice has a larger sum."""
    g = np.random.default_rng(5)
    for _ in range(20):
        s = np.round(g.random(8) * 4) / 4
        rows = kept_rows(s.tolist(), 5, 1, 2)
        best = max(sum(s[list(c)]) for c in itertools.combinations(range(8), 5) if {0, 6, 7} <= set(c))
        assert {0, 6, 7} <= set(rows) and len(rows) == 5 and s[rows].sum() == best


def test_evict_moves_rows_and_leaves_the_rest():
    k = np.arange(2 * 6 * 2, dtype=np.float64).reshape(1, 2, 1, 6, 2)
    score = np.array([[[[3.0, 0, 2, 1, 9, 9]], [[1.0, 2, 3, 9, 9, 9]]]])
    kk, vv, ss, n, idx = oracle.kv_evict(k, -k, score, [4, 3], 3)
    assert n.tolist() == [3, 3] and idx[0, :, 0].tolist() == [[0, 2, 3], [0, 1, 2]]
    assert kk[0, 0, 0, :, 0].tolist() == [0, 4, 6, 6, 8, 10] and (vv == -kk).all()
    assert ss[0, 0, 0].tolist() == [3, 2, 1, 1, 9, 9]
    assert (kk[0, 1] == k[0, 1]).all()
