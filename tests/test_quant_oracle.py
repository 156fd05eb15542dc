"""Pins of the 8-bit cache's oracle: e4m3 against torch's conversion, scales and
block selection against hand values and definitions."""

import itertools
import math

import numpy as np
import pytest
import torch

import oracle as O
from oracle import quant_oracle as Q


def test_e4m3_table_and_rounding_match_torch():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(Q.TABLE, t, equal_nan=True)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(4000) * 10.0 ** rng.uniform(-4, 2, 4000),
                        Q.TABLE[:127], (Q.TABLE[:126] + Q.TABLE[1:127]) / 2, [2.0 ** -10, 448.0]])
    x = np.clip(np.concatenate([x, -x]), -448, 448).astype(np.float32).astype(np.float64)
    want = torch.tensor(x, dtype=torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(Q.to_e4m3(x), want)


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (225.0, 0),
                                    (1.0, -8), (1.75, -8), (1.76, -7), (0.0, -100), (1e-38, -100),
                                    (3.4e38, 120)])
def test_block_exponent(amax, e):
    assert Q.block_exponent(amax) == e


def test_store_block_grows_its_scale_only():
    old, s = Q.store_block(np.zeros((0, 2), np.uint8), 1.0, [[1.0, -1.75]])
    assert s == 2.0 ** -8 and Q.TABLE[old].tolist() == [[256.0, -448.0]]
    # a smaller token keeps the scale, a larger one doubles it and halves what is there
    b1, s1 = Q.store_block(old, s, [[0.5, 0.25]])
    assert s1 == s and Q.TABLE[b1[1]].tolist() == [128.0, 64.0] and np.array_equal(b1[:1], old)
    b2, s2 = Q.store_block(b1, s1, [[3.0, 0.0]])
    assert s2 == 2 * s and (Q.TABLE[b2] * s2).tolist() == [[1.0, -1.75], [0.5, 0.25], [3.0, 0.0]]


def test_scores_bound_every_key():
    rng = np.random.default_rng(1)
    K, Qg = rng.standard_normal((16, 8)), rng.standard_normal((3, 8))
    lo, hi = Q.block_bounds(K)
    s = Q.block_scores(Qg, lo[None], hi[None])[0]
    assert s >= (K @ Qg.T).max()
    # attained by the key of the worst corner
    assert s == pytest.approx(max(sum(max(a * x, b * x) for a, b, x in zip(lo, hi, q)) for q in Qg))


def test_choice_is_the_best_subset_and_ties_go_low():
    sigma = [3.0, 5.0, 5.0, 1.0, 5.0]
    assert Q.choose_blocks(sigma, [0, 1, 2, 3, 4], 32, 16) == [1, 2]
    assert Q.choose_blocks(sigma, [2, 3, 4], 1, 16) == [2]
    assert Q.choose_blocks(sigma, [0, 1], 0, 16) == [] and Q.choose_blocks(sigma, [], 99, 16) == []
    for k in range(1, 5):
        got = sum(sigma[j] for j in Q.choose_blocks(sigma, range(5), 16 * k, 16))
        assert got == max(sum(c) for c in itertools.combinations(sigma, k))


def test_sets_of_blocks_by_hand():
    assert Q.candidate_blocks(100, 4, 10, 16) == [0, 1, 2, 3, 4, 5]
    assert Q.candidate_blocks(100, 16, 20, 16) == [1, 2, 3, 4]
    assert Q.candidate_blocks(20, 16, 10, 16) == []
    S = Q.block_set([0, 5], 100, 4, 10, 16)
    assert S == list(range(16)) + list(range(80, 100))
    assert Q.block_set([], 5, 4, 10, 16) == [0, 1, 2, 3, 4]
    # every block chosen: dense attention
    n, d = 50, 4
    rng = np.random.default_rng(2)
    K, V, q = rng.standard_normal((n, d)), rng.standard_normal((n, d)), rng.standard_normal(d)
    S = Q.block_set(Q.choose_blocks(np.zeros(4), Q.candidate_blocks(n, 4, 3, 16), 999, 16), n, 4, 3, 16)
    y, l = O.sparse_attention(q, K, V, S)
    yd, ld = O.dense_attention(q, K, V)
    assert np.abs(y - yd).max() < 1e-15 and abs(l - ld) < 1e-13
    assert math.isfinite(l)
