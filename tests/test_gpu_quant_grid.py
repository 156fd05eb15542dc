"""Calls of the 8-bit cache and the blocks with millions of units: the last and
the first of them get what a small call gives."""

import pytest
import torch

from paper_2602_08329_amd import binding as B
from tests.test_gpu_quant import DEV, E4, I32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def test_a_store_and_bounds_of_four_million_blocks():
    # of 2^18 sequences three store a token, each on a page of its own
    batch, hkv, d, bs = 1 << 18, 8, 64, 16
    who = [0, batch // 2 + 1, batch - 1]
    table = torch.full((batch, 2), -1, dtype=I32, device=DEV)
    lens, new = (torch.zeros(batch, dtype=I32, device=DEV) for _ in range(2))
    for i, b in enumerate(who):
        table[b, 1], lens[b], new[b] = i, 17, 1
    k1, v1 = (torch.randn(3, hkv, 1, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(i)).bfloat16()
              for i in range(2))
    k, v = (torch.zeros(batch, hkv, 1, d, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    k[who], v[who] = k1, v1

    def stored(table, lens, new, k, v):
        pages = 4
        K, V = (torch.full((pages, hkv, bs, d), 127, dtype=torch.uint8, device=DEV) for _ in "kv")
        ks, vs = (torch.full((pages, hkv), 7.0, device=DEV) for _ in "kv")
        kv = B.QuantKV(K.view(E4), V.view(E4), ks, vs, lens, 32, hkv, table)
        lo, hi = (torch.zeros(pages, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        B.prhs_quant_store(kv, k, v, new, B.BlockBounds(kv, lo, hi))
        X = torch.zeros(pages, hkv, bs, d, dtype=torch.bfloat16, device=DEV)
        X[:, :, 0] = torch.cat([k1, k1[:1]])[:, :, 0]
        plain = B.KV(X, X, lens, 32, hkv, table)
        a, z = (torch.zeros(pages, hkv, d, dtype=torch.bfloat16, device=DEV) for _ in "kv")
        B.prhs_block_bounds(plain, B.BlockBounds(plain, a, z), 32, new)
        return K, V, ks, vs, lo, hi, a, z

    big = stored(table, lens, new, k, v)
    one = torch.tensor([[-1, 0], [-1, 1], [-1, 2]], dtype=I32, device=DEV)
    small = stored(one, lens[who].contiguous(), new[who].contiguous(), k1, v1)
    for x, y in zip(big, small):
        assert torch.equal(x, y)
    assert (big[0][3] == 127).all() and (big[2][3] == 7).all()   # the page that no sequence has


def test_a_selection_of_two_million_rows():
    batch, hkv, d, bs, n = 1 << 18, 8, 64, 16, 64
    pages = 64
    g = torch.Generator(device=DEV).manual_seed(3)
    lo = torch.randn(pages, hkv, d, generator=g, device=DEV).mul_(16).round_().div_(16).bfloat16()
    hi = lo + 1
    table = torch.randint(0, pages, (batch, 16), generator=g, dtype=I32, device=DEV)
    lens = torch.randint(0, 257, (batch,), generator=g, dtype=I32, device=DEV)
    q = torch.randn(batch, hkv, d, generator=g, device=DEV).mul_(16).round_().div_(16).bfloat16()
    X = torch.zeros(pages, hkv, bs, d, dtype=torch.uint8, device=DEV).view(E4)
    sc = torch.ones(pages, hkv, device=DEV)
    p = B.params(k=n, sink=4, window=8)

    def chosen(table, lens, q):
        kv = B.QuantKV(X, X, sc, sc, lens, 256, hkv, table)
        bounds = B.BlockBounds(kv, lo, hi)
        m = len(lens)
        blk, st = (torch.full((m, hkv, c), -9, dtype=I32, device=DEV) for c in (4, 4 + 64 + 8))
        bl, sl = (torch.full((m, hkv), -9, dtype=I32, device=DEV) for _ in range(2))
        ws = B.workspace(B.prhs_block_workspace_size(kv, bounds), DEV)
        B.prhs_block_select(kv, q, p, bounds, blk, bl, st, sl, ws)
        return blk, bl, st, sl

    big = chosen(table, lens, q)
    for s in (slice(0, 2000), slice(batch - 2000, batch), slice(batch // 2, batch // 2 + 2000)):
        for x, y in zip(big, chosen(table[s], lens[s], q[s])):
            assert torch.equal(x[s], y)
