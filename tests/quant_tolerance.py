"""How far attention over an 8-bit cache may be from its definition in 64 bits.

With u = 2^-24, a logit x = scale sum_d q_d k_d is off by at most
dx = (d + 8) u scale sum_d |q_d k_d| + 4 u |x| (fp32 products and sums, scale
factors, the exponent's argument), a weight by dx and 2^-21 relative (the
exponential, its fp16 pair), and fp32 sums of at most n / 32 + 64 terms by as
many u.  y is off by at most twice the weights' relative error times max |v|, lse
by the weights' relative error and 4 u |lse|."""

import numpy as np

U = 2.0 ** -24


def weight_error(q, K, scale):
    """Relative error of the weights of query q over the keys K [n][d]."""
    n, d = K.shape
    x = np.abs(K @ q) * scale
    dx = ((d + 8) * U * scale * (np.abs(K) @ np.abs(q))).max() + 4 * U * x.max()
    return dx + 2.0 ** -21 + (n / 32 + 64) * U


def assert_attention(y, lse, yr, lr, q, K, V, scale, what=""):
    rel = weight_error(q, K, scale)
    off, may = np.abs(y - yr).max(), 2 * rel * np.abs(V).max()
    assert off <= may, (what, off, may)
    assert abs(lse - lr) <= rel + 4 * U * abs(lr), (what, lse, lr)
