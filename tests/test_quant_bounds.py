"""What a block's score says about its keys: those as given never exceed it, and
those an 8-bit cache stores by no more than their rounding."""

import numpy as np
import pytest

from oracle import quant_oracle as Q


def stored(keys, chunks):
    """A block's keys as the cache holds them, its final scale, and its bounds,
    stored in chunks of the given sizes."""
    raw, s = np.zeros((0, keys.shape[1]), np.uint8), 1.0
    at = 0
    for c in chunks:
        raw, s = Q.store_block(raw, s, keys[at: at + c])
        at += c
    return Q.TABLE[raw] * s, s, Q.block_bounds(keys)


def slack(q, lo, hi, s):
    """How far a stored key may exceed the score: half a step of each element, and
    what growing scales add below 2^-6 of the last, 2^-10 s (1 + 1/2 + ..)."""
    return (np.abs(q) * (2.0 ** -4 * np.maximum(np.abs(lo), np.abs(hi)) + 2.0 ** -9 * s)).sum(1).max()


@pytest.mark.parametrize("chunks", [[16], [1] * 16, [5, 1, 10]])
@pytest.mark.parametrize("wide", [0.0, 6.0])
def test_stored_keys_exceed_a_score_by_their_rounding_only(chunks, wide):
    rng = np.random.default_rng(len(chunks))
    over = 0
    for _ in range(100):
        keys = rng.standard_normal((16, 32)) * 2.0 ** rng.uniform(-wide, wide, (16, 1))
        q = rng.standard_normal((3, 32))
        k8, s, (lo, hi) = stored(keys, chunks)
        sigma = Q.block_scores(q, lo[None], hi[None])[0]
        assert (keys @ q.T).max() <= sigma
        best = (k8 @ q.T).max()
        assert best <= sigma + slack(q, lo, hi, s)
        out = (k8 < lo) | (k8 > hi)
        over += out.any()
    assert over > 50   # elements do leave the bounds


def test_a_stored_key_above_its_block_s_score():
    # the scale is 1/16, 280 of it lies between 256 and 288: 17.5 is stored as 18
    keys, q = np.full((16, 64), 17.5), np.ones((1, 64))
    k8, s, (lo, hi) = stored(keys, [16])
    sigma = Q.block_scores(q, lo[None], hi[None])[0]
    assert sigma == 1120 and (k8 @ q.T).max() == 1152 <= sigma + slack(q, lo, hi, s)
