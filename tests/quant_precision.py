"""Inputs on which attention over an 8-bit cache shows how many bits it keeps of
a query and of a weight, and how far each result may be off.  Keys and values
have one element that is not zero: a key's gives its logit as a single product,
a value's row is the only one that carries its dim, so no sum hides an error.

With u = 2^-24, a logit x = scale ks q k8 in fp32: one rounding each of the
product q k8, scale, scale log2(e) (the constant's too), ks times that, their
product, and the way back to base e (two): |dx| <= 8 u |x|.  A weight exp(x - m):
dx, 1 u |x| of the subtraction and two units of the exponential, p vs, its parts
(24 bits) and one unit a joining of waves and of splits, 8 u in all with the
final division.  Its sum over n tokens: a lane of four or eight waves adds at
most n / 16, the joinings 16 more."""

import numpy as np

from oracle import quant_oracle as Q

U = 2.0 ** -24


def logit_tolerance(x):
    return 8 * U * np.abs(x)


def weight_tolerance(x):
    """Relative, of exp(x_i) / sum exp(x): both sides of the quotient."""
    return (2 * (9 * np.abs(x).max() + 8) + len(x) / 16 + 16) * U


def bf16(x):
    """fp32 values rounded to bf16, ties to even."""
    b = np.asarray(x, np.float32).view(np.uint32).astype(np.uint64)
    b = (b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000
    return b.astype(np.uint32).view(np.float32)


def parts(x, count, rnd):
    """x as the sum of `count` numbers of fewer bits, each the rest rounded."""
    rest, s = np.asarray(x, np.float32), np.zeros(np.shape(x))
    for _ in range(count):
        h = rnd(rest).astype(np.float32)
        s += h.astype(np.float64)
        rest = rest - h
    return s


def queries(rng, shape):
    """fp32 values of which two bf16 parts (8 bits each) leave as much as they can:
    63 of 2^23 to 2^24."""
    m = (rng.integers(128, 256, shape) << 16) + (rng.integers(128, 255, shape) << 7) + 63
    return (m * 2.0 ** -23 * rng.choice([-1.0, 1.0], shape)).astype(np.float32)


class Unit:
    """One (batch, kv head): key bytes, value bytes and scales of n rows, the
    dim of each key (kd) and the row that carries each dim of the values (vr).
    Block `big` of the values has a scale 2^spread times the others'."""

    def __init__(self, rng, n, d, bs, spread=0, big=0):
        m = -(-n // bs)
        self.n, self.d = n, d
        self.k, self.v = (np.zeros((m * bs, d), np.uint8) for _ in "kv")
        self.kd, self.vr = rng.integers(0, d, n), rng.permutation(n)[np.arange(d) % n]
        self.k[np.arange(n), self.kd] = rng.integers(0x30, 0x41, n) + 128 * rng.integers(0, 2, n)
        self.v[self.vr, np.arange(d)] = rng.integers(0x30, 0x7F, d) + 128 * rng.integers(0, 2, d)
        self.ks = np.full(m, 2.0 ** rng.integers(-1, 2), np.float32)
        self.vs = np.full(m, np.float32(2.0 ** -3 * 1.25))
        self.vs[big % m] *= 2.0 ** spread
        self.bs = bs

    def logits(self, q, scale):
        r = np.arange(self.n)
        return scale * self.ks.astype(float)[r // self.bs] * q.astype(float)[self.kd] * Q.TABLE[self.k[r, self.kd]]

    def output(self, x):
        """y and lse of logits x, in 64 bits."""
        w = np.exp(x - x.max())
        v = Q.TABLE[self.v[self.vr, np.arange(self.d)]] * self.vs.astype(float)[self.vr // self.bs]
        return w[self.vr] * v / w.sum(), x.max() + np.log(w.sum())


def off_by(y, lse, yr, lr, x):
    """Largest error in units of what is allowed, of y (every dim by itself) and lse."""
    return (np.abs(y / yr - 1).max() / weight_tolerance(x),
            abs(lse - lr) / (weight_tolerance(x) + logit_tolerance(lr)))
