"""Attention over an 8-bit cache whose attended rows hold NaN (as the store
writes for NaN and infinite elements), and NaN queries: they reach exactly the
outputs that depend on them."""

import math

import numpy as np
import pytest
import torch

from paper_2602_08329_amd import binding as B
from tests.test_gpu_quant import DEV, I32, Cache, Store, dense, pack

pytestmark = pytest.mark.gpu
NAN = 127   # the byte


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


# (lengths, q heads, kv heads, d, paged, dtype): whole units, split ones, more than eight heads a kv head
CASES = [
    ((200, 90), 4, 2, 128, True, "bf16"),
    ((6000, 5200), 4, 2, 128, True, "bf16"),
    ((300, 40), 18, 2, 64, False, "f32"),
    ((5000, 4100), 16, 1, 64, False, "f32"),
    ((2500, 1700), 3, 1, 128, False, "f32"),
]


def attend(c, form):
    """One call over every token, as a dense stream or as sets of all positions."""
    if form == "dense":
        return dense(c)
    cap, Bn = max(c.lens), len(c.lens)
    rng = np.random.default_rng(1)
    sets = {(b, g): rng.permutation(n) for b, n in enumerate(c.lens) for g in range(c.hkv)}
    idx, ln = pack(sets, Bn, c.hkv, cap)
    y, lse = c.outputs()
    B.prhs_quant_sparse_decode_attn(c.kv, c.q, idx, ln, c.scale_q, y, lse, c.workspace(False, cap))
    return y, lse


def put(c, x, b, g, pos, dims):
    """NaN into the dims of position pos of a unit's K or V."""
    t = c.dev[x].view(torch.uint8)
    i = c.block(b, g, pos // c.bs)
    t.view(-1, c.bs, c.d)[i, pos % c.bs, dims] = NAN


def same(a, b):
    return torch.equal(a, b) and bool(torch.isfinite(a).all())


@pytest.mark.parametrize("form", ["dense", "sparse"])
@pytest.mark.parametrize("lens,hq,hkv,d,paged,dtype", CASES)
def test_nan_reaches_what_attends_it(lens, hq, hkv, d, paged, dtype, form):
    c = Cache(lens, hq, hkv, d, 16, paged, dtype, seed=lens[0])
    G = hq // hkv
    y0, l0 = attend(c, form)
    # a NaN element of one key: every head of its unit, all dims and lse
    for pos in {0, lens[1] // 2, lens[1] - 1}:
        c = Cache(lens, hq, hkv, d, 16, paged, dtype, seed=lens[0])
        put(c, "k", 1, hkv - 1, pos, slice(5, 6))
        y, lse = attend(c, form)
        hit = slice((hkv - 1) * G, hkv * G)
        assert y[1, hit].isnan().all() and lse[1, hit].isnan().all(), pos
        assert same(y[0], y0[0]) and same(lse[0], l0[0])
        assert same(y[1, : hit.start], y0[1, : hit.start]) and same(lse[1, : hit.start], l0[1, : hit.start])
    # of one value: its dim alone, and lse is what it was
    c = Cache(lens, hq, hkv, d, 16, paged, dtype, seed=lens[0])
    put(c, "v", 0, 0, lens[0] // 2, slice(7, 8))
    y, lse = attend(c, form)
    assert torch.equal(lse, l0) and y[0, :G, 7].isnan().all()
    y[0, :G, 7] = y0[0, :G, 7]
    assert same(y, y0)
    # of one query: its head alone
    c = Cache(lens, hq, hkv, d, 16, paged, dtype, seed=lens[0])
    c.q[0, hq - 1, 3] = math.nan
    y, lse = attend(c, form)
    assert y[0, hq - 1].isnan().all() and lse[0, hq - 1].isnan()
    assert same(y[0, : hq - 1], y0[0, : hq - 1]) and same(y[1], y0[1]) and same(lse[1], l0[1])


@pytest.mark.parametrize("n", [70, 5000])
def test_nothing_but_nan_keys(n):
    # every logit of every split is NaN; and no token at all stays y = 0, lse = -inf
    c = Cache((n, 0), 4, 2, 64, 16, True, "bf16", seed=n)
    for pos in range(n):
        put(c, "k", 0, 1, pos, slice(0, 1))
    y, lse = attend(c, "dense")
    assert y[0, 2:].isnan().all() and lse[0, 2:].isnan().all()
    assert y[0, :2].isfinite().all() and lse[0, :2].isfinite().all()
    assert (y[1] == 0).all() and (lse[1] == -math.inf).all()


def test_an_infinite_key_that_was_stored():
    # the store keeps it as NaN, which attention gives; a set without it does not
    s = Store(1, 1, 64, 16, True, "bf16", 48, seed=3)
    k, v = s.tokens(40, wide=0.0)
    k[0, 0, 20, 9] = -math.inf
    s.store(k, v)
    s.check()
    s.c.lens = (40,)
    y, lse = dense(s.c)
    assert y.isnan().all() and lse.isnan().all()
    idx, ln = pack({(0, 0): [p for p in range(40) if p != 20]}, 1, 1, 40)
    y, lse = s.c.outputs()
    B.prhs_quant_sparse_decode_attn(s.c.kv, s.c.q, idx, ln, s.c.scale_q, y, lse, s.c.workspace(False, 40))
    s.c.check(y, lse, lambda b, g: [p for p in range(40) if p != 20])
    one = torch.tensor([[1]], dtype=I32, device=DEV)
    y, lse = s.c.outputs()
    B.prhs_quant_sparse_decode_attn(s.c.kv, s.c.q, torch.full((1, 1, 40), 20, dtype=I32, device=DEV), one, s.c.scale_q,
                                    y, lse, s.c.workspace(False, 40))
    assert y.isnan().all() and lse.isnan().all()
