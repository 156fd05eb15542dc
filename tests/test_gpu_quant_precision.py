"""How many bits attention over an 8-bit cache keeps of queries and weights, on
inputs whose sums hide no error (quant_precision), every dim by itself."""

import numpy as np
import pytest
import torch

from paper_2602_08329_amd import binding as B
from tests import quant_precision as P
from tests.test_gpu_quant import DEV, I32, Cache, dense

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def cache(units, lens, hq, hkv, d, paged, dtype, q):
    """A Cache that holds the given units, and its queries."""
    bs = next(iter(units.values())).bs
    c = Cache(lens, hq, hkv, d, bs, paged, dtype, fill=False)
    for (b, g), u in units.items():
        for j in range(-(-u.n // bs)):
            i, r = c.block(b, g, j), min(bs, u.n - j * bs)
            for x, t, s in (("k", u.k, u.ks), ("v", u.v, u.vs)):
                c.raw[x][i, :r], c.scale[x][i] = t[j * bs: j * bs + r], s[j]
    for x in "kv":
        c.dev[x].view(torch.uint8).copy_(torch.tensor(c.raw[x]).view(c.dev[x].shape))
        c.dsc[x].copy_(torch.tensor(c.scale[x]).view(c.dsc[x].shape))
    c.q = torch.tensor(q).to(c.dtype).to(DEV)
    return c


@pytest.mark.parametrize("d,hq,hkv", [(64, 8, 1), (128, 4, 2), (64, 16, 1), (128, 9, 1)])
def test_fp32_queries_keep_their_bits(d, hq, hkv):
    # one token a sequence: lse is its logit, a single product
    rng = np.random.default_rng(d + hq)
    lens = (1,) * 24
    units = {(b, g): P.Unit(rng, 1, d, 16) for b in range(24) for g in range(hkv)}
    q = P.queries(rng, (24, hq, d)) * np.float32(16)
    c = cache(units, lens, hq, hkv, d, False, "f32", q)
    y, lse = dense(c)
    lse, G = lse.double().cpu().numpy(), hq // hkv
    for (b, g), u in units.items():
        for h in range(g * G, (g + 1) * G):
            x = u.logits(q[b, h], float(np.float32(c.scale_q)))
            assert abs(lse[b, h] - x[0]) <= P.logit_tolerance(x[0]), (b, h)


@pytest.mark.parametrize("spread", [0, 16, 40, 100])
@pytest.mark.parametrize("n,d,hq,hkv,paged,dtype", [
    (48, 128, 4, 2, True, "bf16"), (130, 64, 16, 1, False, "bf16"), (700, 128, 8, 1, True, "f32"),
    (5000, 64, 4, 1, False, "bf16"), (130, 128, 10, 1, True, "f32"), (2048, 128, 9, 1, False, "bf16"),
])
def test_weights_keep_their_bits_whatever_the_scales(n, d, hq, hkv, paged, dtype, spread):
    # a block of far larger values stands first, in the middle or last; the dims
    # that it does not carry are as exact as without it, as sets too
    rng = np.random.default_rng(n + spread)
    m = -(-n // 16)
    lens = (n, n - 7, n)
    units = {(b, g): P.Unit(rng, lens[b], d, 16, spread, big=(0, m // 2, m - 1)[b]) for b in range(3) for g in range(hkv)}
    q = rng.standard_normal((3, hq, d)).astype(np.float32)
    q = P.bf16(q) if dtype == "bf16" else q
    c = cache(units, lens, hq, hkv, d, paged, dtype, q)
    got = [dense(c)]
    idx = torch.arange(n, dtype=I32, device=DEV).flip(0).expand(3, hkv, n).contiguous()
    y, lse = c.outputs()
    B.prhs_quant_sparse_decode_attn(c.kv, c.q, idx, torch.full((3, hkv), n, dtype=I32, device=DEV), c.scale_q, y, lse,
                                    c.workspace(False, n))
    got.append((y, lse))
    G = hq // hkv
    for y, lse in got:
        y, lse = y.double().cpu().numpy(), lse.double().cpu().numpy()
        for (b, g), u in units.items():
            for h in range(g * G, (g + 1) * G):
                x = u.logits(q[b, h], float(np.float32(c.scale_q)))
                off = P.off_by(y[b, h], lse[b, h], *u.output(x), x)
                assert max(off) <= 1, (b, h, off)
