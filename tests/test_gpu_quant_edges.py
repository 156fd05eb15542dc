"""The 8-bit cache's and the blocks' calls at their smallest, and in two graphs
that share a workspace."""

import math

import pytest
import torch

from paper_2602_08329_amd import binding as B
from tests.test_gpu_quant import DEV, E4, I32, Cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.lib()


def empty_cache(batch, hkv, d, n, paged):
    nb = max(1, -(-n // 16))
    shape, lead = ((4, hkv, 16, d), (4, hkv)) if paged else ((batch, hkv, nb * 16, d), (batch, hkv, nb))
    K, V = (torch.full(shape, 127, dtype=torch.uint8, device=DEV).view(E4) for _ in "kv")
    ks, vs = (torch.full(lead, math.nan, device=DEV) for _ in "kv")
    table = torch.full((batch, nb), -1, dtype=I32, device=DEV) if paged else None
    kv = B.QuantKV(K, V, ks, vs, torch.zeros(batch, dtype=I32, device=DEV), n, 4 * hkv, table)
    return kv, B.BlockBounds(kv, *(torch.full((*lead, d), 3.0, dtype=torch.bfloat16, device=DEV) for _ in "kv"))


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("batch,n,T", [(0, 32, 2), (3, 0, 2), (3, 32, 0), (3, 32, 2)])
def test_nothing_to_store_or_attend(batch, n, T, paged):
    # no sequence, no room, no new token, no token at all
    hkv, d, cap = 2, 64, 40
    kv, bounds = empty_cache(batch, hkv, d, n, paged)
    before = [t.view(torch.uint8).clone() for t in (*kv._keep[:4], *bounds._keep)]
    new = torch.ones(batch, hkv, T, d, dtype=torch.bfloat16, device=DEV)
    B.prhs_quant_store(kv, new, new, None, bounds)
    for t, x in zip((*kv._keep[:4], *bounds._keep), before):
        assert torch.equal(t.view(torch.uint8), x)
    q = torch.ones(batch, 4 * hkv, d, dtype=torch.bfloat16, device=DEV)
    blk, st = (torch.full((batch, hkv, cap), -9, dtype=I32, device=DEV) for _ in range(2))
    bl, sl = (torch.full((batch, hkv), -9, dtype=I32, device=DEV) for _ in range(2))
    ws = B.workspace(max(B.prhs_block_workspace_size(kv, bounds), B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, kv),
                         B.prhs_workspace_size(B.PRHS_OP_QUANT_SPARSE_ATTN, kv, None, cap)), DEV)
    B.prhs_block_select(kv, q, B.params(k=16, sink=4, window=4), bounds, blk, bl, st, sl, ws)
    assert (bl == 0).all() and (sl == 0).all() and (st == -9).all() and (blk == -9).all()
    sl.fill_(cap)   # entries that name no position
    for call in (lambda y, s: B.prhs_quant_dense_decode_attn(kv, q, 0.1, y, s, ws),
                 lambda y, s: B.prhs_quant_sparse_decode_attn(kv, q, st, sl, 0.1, y, s, ws)):
        y, lse = torch.full(q.shape, 7.0, device=DEV), torch.full(q.shape[:2], 7.0, device=DEV)
        call(y, lse)
        assert (y == 0).all() and (lse == -math.inf).all()


def test_two_graphs_that_share_a_workspace():
    # split units of 16 heads of d 128, more than 48 KB of LDS a workgroup; replayed
    # in any order, with eager calls that leave other partials in the workspace
    c = Cache((5000, 3100), 32, 2, 128, 16, True, "f32", seed=50)
    e = Cache((9000,), 8, 2, 128, 32, False, "bf16", seed=51)
    n = max(B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, x.kv) for x in (c, e))
    ws = B.workspace(n, DEV)
    outs, want, graphs = [x.outputs() for x in (c, e)], [], []
    for x, (y, lse) in zip((c, e), outs):
        B.prhs_quant_dense_decode_attn(x.kv, x.q, x.scale_q, y, lse, ws)
        want.append((y.clone(), lse.clone()))
    torch.cuda.synchronize()
    for x, (y, lse) in zip((c, e), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            B.prhs_quant_dense_decode_attn(x.kv, x.q, x.scale_q, y, lse, ws)
    for order in ((0, 1), (1, 0), (0, 0, 1)):
        for y, lse in outs:
            y.zero_(), lse.zero_()
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for (y, lse), (yw, lw) in zip(outs, want):
            assert torch.equal(y, yw) and torch.equal(lse, lw)
        ws.fill_(255)
        torch.randn(1000, device=DEV).sum().item()
