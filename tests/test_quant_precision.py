"""The precision inputs tell schemes apart: emulated in NumPy, three bf16 parts
of a query and of a weight pass, and fewer or narrower parts do not."""

import numpy as np
import pytest

from oracle import quant_oracle as Q
from tests import quant_precision as P


@pytest.mark.parametrize("count,passes", [(1, False), (2, False), (3, True)])
def test_bits_of_a_query(count, passes):
    rng = np.random.default_rng(0)
    q = P.queries(rng, 64)
    u = P.Unit(rng, 1, 64, 16)
    x, got = (np.array([Q.TABLE[0x40] * v for v in w]) for w in (q.astype(float), P.parts(q, count, P.bf16)))
    assert u.logits(q, 1.0).shape == (1,)
    assert (np.abs(got - x) <= P.logit_tolerance(x)).any() == passes
    assert (np.abs(got - x) <= P.logit_tolerance(x)).all() == passes


def emulate(u, x, split):
    """y from weights p vs r held as split(.) holds them, r bringing the largest
    scale to [2^6, 2^7) as a scheme in fp16 does, or to 2^80."""
    p = np.exp2(((x - x.max()) * np.log2(np.e)).astype(np.float32))
    vs = u.vs[u.vr // u.bs]
    top = np.floor(np.log2(u.vs.max()))
    r = 2.0 ** ((80 if split == "bf16 x 3" else 6) - top)
    w = p[u.vr] * (vs.astype(np.float64) * r).astype(np.float32)
    w = {"bf16 x 3": lambda: P.parts(w, 3, P.bf16), "bf16 x 2": lambda: P.parts(w, 2, P.bf16),
         "f16 x 2": lambda: P.parts(w, 2, np.float16), "f16": lambda: P.parts(w, 1, np.float16)}[split]()
    return w / r * Q.TABLE[u.v[u.vr, np.arange(u.d)]] / p.astype(np.float64).sum()


@pytest.mark.parametrize("spread", [0, 16, 24, 40, 100])
@pytest.mark.parametrize("n", [48, 130])
def test_bits_of_a_weight(n, spread):
    rng = np.random.default_rng(n + spread)
    u = P.Unit(rng, n, 128, 16, spread, big=1)
    x = u.logits(rng.standard_normal(128).astype(np.float32), 128 ** -0.5)
    yr, lr = u.output(x)

    def ok(split):
        return P.off_by(emulate(u, x, split), lr, yr, lr, x)[0] <= 1

    assert ok("bf16 x 3") and not ok("bf16 x 2") and not ok("f16")
    assert ok("f16 x 2") == (spread == 0)


def test_output_of_a_unit_is_attention():
    rng = np.random.default_rng(4)
    u = P.Unit(rng, 37, 64, 16, 3, big=2)
    q = rng.standard_normal(64).astype(np.float32)
    r = np.arange(u.n)
    K, V = (Q.TABLE[t[: u.n]] * s.astype(float)[r // u.bs][:, None] for t, s in ((u.k, u.ks), (u.v, u.vs)))
    x = 0.125 * (K @ q.astype(float))
    w = np.exp(x - x.max())
    y, lse = u.output(u.logits(q, 0.125))
    assert np.allclose(y, w @ V / w.sum(), rtol=1e-12, atol=0) and abs(lse - x.max() - np.log(w.sum())) < 1e-12
