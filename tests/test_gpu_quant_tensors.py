"""The 8-bit cache's and the blocks' calls on tensors that are aligned to their
elements only, on other streams and from several threads: what the same calls
give on tensors of their own, on the current stream, one after another."""

import threading

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


def plain(*shape, dtype):
    return torch.zeros(*shape, dtype=dtype, device=DEV)


def shifted(*shape, dtype):
    """A contiguous tensor that begins one element behind an aligned address."""
    n = 1
    for s in shape:
        n *= s
    t = torch.zeros(n + 1, dtype=dtype, device=DEV)[1:].view(shape)
    assert t.data_ptr() % 16 == torch.tensor([], dtype=dtype).element_size()
    return t


def decode(seed, dtype, paged, d=64, hq=10, hkv=2, new=plain, stream=None):
    """A prompt and two steps: store, bounds, selection and every attention; all
    outputs and the cache.  `new` makes the tensors that need no alignment."""
    bs, batch, n, T = 16, 3, 700, 3
    g = torch.Generator(device=DEV).manual_seed(seed)
    nb = -(-(n + T) // bs)
    lead = (batch * nb, hkv) if paged else (batch, hkv, nb)
    K, V = (plain(*((batch * nb, hkv, bs, d) if paged else (batch, hkv, nb * bs, d)), dtype=torch.uint8) for _ in "kv")
    ks, vs = new(*lead, dtype=torch.float32), new(*lead, dtype=torch.float32)
    lo, hi = (plain(*lead, d, dtype=dtype) for _ in "kv")
    lens, anchor = new(batch, dtype=I32), new(batch, dtype=I32)
    table = None
    if paged:
        table = new(batch, nb, dtype=I32)
        table.copy_(torch.randperm(batch * nb, generator=g, device=DEV).view(batch, nb))
    kv = B.QuantKV(K.view(E4), V.view(E4), ks, vs, lens, n + T, hq, table, dtype=dtype)
    bounds = B.BlockBounds(kv, lo, hi)
    p = B.params(k=100, sink=4, window=20, refresh_every=T)
    kc, sc = B.prhs_max_blocks(p, bs, n + T), B.prhs_block_set_capacity(p, bs, n + T)
    blk, st = new(batch, hkv, kc, dtype=I32), new(batch, hkv, sc, dtype=I32)
    bl, sl = new(batch, hkv, dtype=I32), new(batch, hkv, dtype=I32)
    ws = B.workspace(max(B.prhs_block_workspace_size(kv, bounds),
                         B.prhs_workspace_size(B.PRHS_OP_QUANT_SPARSE_ATTN, kv, None, sc),
                         B.prhs_workspace_size(B.PRHS_OP_QUANT_DENSE_ATTN, kv)), DEV)
    res = []

    tail, ids = new(batch * hkv, dtype=I32), new(batch * hkv, dtype=I32)
    ids.copy_(torch.arange(batch * hkv, device=DEV))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    at = stream or torch.cuda.current_stream()

    def out():
        with torch.cuda.stream(at):
            res.append((new(batch, hq, d, dtype=torch.float32), new(batch, hq, dtype=torch.float32)))
        return res[-1]

    for t in range(T):
        m = n if t == 0 else 1
        with torch.cuda.stream(at):   # the inputs; the calls are told their stream
            k, v, q = (new(batch, hkv, m, d, dtype=dtype), new(batch, hkv, m, d, dtype=dtype), new(batch, hq, d, dtype=dtype))
            for x in (k, v, q):
                x.copy_(torch.randn(x.shape, generator=g, device=DEV).mul_(16).round_().div_(16))
            nl = new(batch, dtype=I32)
            nl.copy_(torch.tensor([m, m - m // 3, m], device=DEV))
            lens.add_(nl)
            if t == 0:
                anchor.copy_(lens)
                tail.copy_(lens.repeat_interleave(hkv))
        B.prhs_quant_store(kv, k, v, nl, bounds, stream=stream)
        if t == 0:
            B.prhs_block_select(kv, q, p, bounds, blk, bl, st, sl, ws, stream=stream)
        B.prhs_quant_sparse_decode_attn(kv, q, st, sl, 0.1, *out(), ws, stream=stream)
        B.prhs_quant_reuse_decode_attn(kv, q, st, sl, anchor, 0.1, *out(), ws, stream=stream)
        B.prhs_quant_pool_decode_attn(kv, q, st, sl, ids, tail, 0.1, *out(), ws, stream=stream)
        B.prhs_quant_dense_decode_attn(kv, q, 0.1, *out(), ws, stream=stream)
        with torch.cuda.stream(at):
            X = plain(*K.shape, dtype=dtype)
            X.copy_(K.float())
            a, z = (plain(*lead, d, dtype=dtype) for _ in "kv")
        other = B.KV(X, X, lens, n + T, hq, table)
        B.prhs_block_bounds(other, B.BlockBounds(other, a, z), n, nl, stream=stream)
        res.append((a, z))
    at.synchronize()
    return [x for pair in res for x in pair] + [K, V, ks, vs, lo, hi, blk, bl, st, sl]


CASES = [(1, torch.bfloat16, True, 64), (2, torch.float32, False, 128), (3, torch.float32, True, 64), (4, torch.bfloat16, False, 128)]


@pytest.mark.parametrize("seed,dtype,paged,d", CASES)
def test_tensors_aligned_to_their_elements(seed, dtype, paged, d):
    for i, (x, y) in enumerate(zip(decode(seed, dtype, paged, d), decode(seed, dtype, paged, d, new=shifted))):
        assert torch.equal(x, y), i


@pytest.mark.parametrize("native", [True, False])
def test_another_stream(native, monkeypatch):
    want = decode(*CASES[0])
    if not native:
        monkeypatch.setattr(B, "_host", None)
    for i, (x, y) in enumerate(zip(want, decode(*CASES[0], stream=torch.cuda.Stream()))):
        assert torch.equal(x, y), i
    with torch.cuda.stream(torch.cuda.Stream()):   # the current one
        got = decode(*CASES[0])
    for i, (x, y) in enumerate(zip(want, got)):
        assert torch.equal(x, y), i


def test_threads_on_streams_of_their_own():
    want = [decode(*c) for c in CASES]
    wrong = []

    def work(i):
        try:
            s = torch.cuda.Stream()
            for _ in range(3):
                for x, y in zip(want[i], decode(*CASES[i], stream=s)):
                    if not torch.equal(x, y):
                        wrong.append(i)
        except Exception as e:   # shown by the assertion
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(CASES))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
