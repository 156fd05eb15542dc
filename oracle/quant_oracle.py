"""Oracle of the block-structured 8-bit KV cache, in fp64: the store, key
bounds of blocks and the selection of whole blocks, one (batch, kv head) unit
at a time.  Attention over the cache is the ordinary attention of
prhs_oracle over the values the cache stands for."""

from __future__ import annotations

import math

import numpy as np

EXP_MIN = -100


def e4m3_table():
    """The 256 values of e4m3 by their bytes (0x7F and 0xFF: NaN)."""
    v = np.empty(256)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        if e == 15 and m == 7:
            v[b] = math.nan
        else:
            x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
            v[b] = -x if s else x
    return v


TABLE = e4m3_table()


def to_e4m3(x):
    """Bytes of the e4m3 values nearest to x (|x| <= 448), ties to the even
    byte; NaN where x is not finite."""
    x = np.asarray(x, dtype=np.float64)
    pos = TABLE[:127]                       # 0 .. 448, ascending
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.clip(hi - 1, 0, 126)
    dl, dh = a - pos[lo], pos[hi] - a
    pick = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    byte = np.where(np.signbit(x), pick + 128, pick)
    return np.where(np.isfinite(x), byte, 127).astype(np.uint8)


def block_exponent(amax):
    """Smallest e >= EXP_MIN with amax <= 448 * 2^e."""
    if not amax > 0:
        return EXP_MIN
    m, e = math.frexp(amax / 448.0)   # division by 7 * 2^6 rounds: settle it below
    e = e - 1
    while 448.0 * math.ldexp(1.0, e) < amax:
        e += 1
    while 448.0 * math.ldexp(1.0, e - 1) >= amax:
        e -= 1
    return max(e, EXP_MIN)


def store_block(old, s_old, new):
    """One block: its earlier elements' bytes `old` [r0][d] under scale s_old,
    then new elements [r1][d].  Returns (bytes [r0 + r1][d], scale)."""
    new = np.asarray(new, dtype=np.float64)
    fin = np.abs(new[np.isfinite(new)])
    need = math.ldexp(1.0, block_exponent(float(fin.max()) if fin.size else 0.0))
    s = need if len(old) == 0 else max(float(s_old), need)
    kept = np.asarray(old, dtype=np.uint8)
    if len(old) and s > s_old:
        kept = to_e4m3(float(s_old) * TABLE[kept] / s)
    return np.concatenate([kept.reshape(-1, new.shape[1]), to_e4m3(new / s)]), s


def block_bounds(keys):
    """Elementwise minimum and maximum of a block's keys [r][d], NaN left out."""
    k = np.asarray(keys, dtype=np.float64)
    return (np.where(np.isnan(k), math.inf, k).min(0), np.where(np.isnan(k), -math.inf, k).max(0))


def block_scores(Qg, k_min, k_max):
    """max over the group's heads of sum_d max(q kmin, q kmax), [blocks]."""
    Qg, lo, hi = (np.asarray(x, dtype=np.float64) for x in (Qg, k_min, k_max))
    return np.max([np.maximum(q * lo, q * hi).sum(1) for q in Qg], axis=0)


def candidate_blocks(n0, sink, window, bs):
    """Blocks that hold a position of the middle range."""
    se = min(sink, n0)
    ws = max(se, n0 - window)
    return sorted({p // bs for p in range(se, ws)})


def choose_blocks(sigma, cand, k_b, bs):
    """The ceil(k_b / bs) candidates of largest sigma, ties to the lower block,
    ascending."""
    rank = sorted(cand, key=lambda j: (-sigma[j], j))
    return sorted(rank[: -(-k_b // bs)])


def block_set(blocks, n0, sink, window, bs):
    """sink U the blocks' positions U window, within [0, n0), ascending."""
    S = set(range(min(sink, n0))) | set(range(max(min(sink, n0), n0 - window), n0))
    for j in blocks:
        S |= set(range(j * bs, min(n0, (j + 1) * bs)))
    return sorted(S)
