"""The 8-bit cache and the block selection on the host: sizes, budgets and
refusals of the C entry points and of the binding (no call here reaches a
launch)."""

import ctypes
import random
import re

import pytest
import torch

from oracle import quant_oracle as Q
from paper_2602_08329_amd import binding as B


@pytest.fixture(scope="module")
def L():
    return B.lib()


def c_kv(**over):
    f = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, dtype=B.PRHS_BF16,
             layout=B.PRHS_KV_CONTIGUOUS, capacity=1024, page_size=16, max_pages=64,
             num_pages=128, k=0x1000, v=0x2000, block_table=0x9000, seq_lens=0x3000,
             max_seq_len=1000)
    f.update(over)
    return B.PrhsKv(**f)


def c_quant(block_size=16, k_scale=0x5000, v_scale=0x6000, **over):
    return B.PrhsQuantKv(c_kv(**over), block_size, k_scale, v_scale)


BAD_QUANT = [
    (dict(block_size=8), B.PRHS_E_UNSUPPORTED, "block_size"),
    (dict(block_size=0), B.PRHS_E_UNSUPPORTED, "block_size"),
    (dict(block_size=256), B.PRHS_E_UNSUPPORTED, "block_size"),
    (dict(capacity=1000), B.PRHS_E_INVALID, "capacity"),
    (dict(layout=B.PRHS_KV_PAGED, page_size=32), B.PRHS_E_INVALID, "page size"),
    (dict(k_scale=None), B.PRHS_E_INVALID, "k_scale"),
    (dict(v_scale=None), B.PRHS_E_INVALID, "v_scale"),
    (dict(k=0x1008), B.PRHS_E_INVALID, "aligned"),
    (dict(v=0x2001), B.PRHS_E_INVALID, "aligned"),
    (dict(k=None), B.PRHS_E_INVALID, "NULL"),
    (dict(seq_lens=None), B.PRHS_E_INVALID, "seq_lens"),
    (dict(head_dim=96), B.PRHS_E_UNSUPPORTED, "head_dim"),
    (dict(num_q_heads=34), B.PRHS_E_UNSUPPORTED, "<= 16"),
    (dict(max_seq_len=2000), B.PRHS_E_INVALID, "capacity"),
    (dict(layout=B.PRHS_KV_PAGED, block_table=None), B.PRHS_E_INVALID, "block_table"),
]


def calls(L, kv, bounds=None, **a):
    """The status of every entry point that takes the cache, with pointers that
    are never read."""
    x, big, ref = 0x10000, 1 << 40, ctypes.byref(kv)
    bd = None if bounds is None else ctypes.byref(bounds)
    return {
        "store": lambda: L.prhs_quant_store(ref, x, x, a.get("new_cap", 1), None, bd, None),
        "sparse": lambda: L.prhs_quant_sparse_decode_attn(ref, x, x, x, a.get("cap", 64), a.get("scale", 1.0), x, None, a.get("ws", x), a.get("bytes", big), None),
        "reuse": lambda: L.prhs_quant_reuse_decode_attn(ref, x, x, x, a.get("cap", 64), a.get("anchor", x), a.get("scale", 1.0), x, None, a.get("ws", x), a.get("bytes", big), None),
        "dense": lambda: L.prhs_quant_dense_decode_attn(ref, x, a.get("scale", 1.0), x, None, a.get("ws", x), a.get("bytes", big), None),
        "pool": lambda: L.prhs_quant_pool_decode_attn(ref, x, x, x, a.get("rows", 4), a.get("cap", 64), a.get("unit", x), x, None, a.get("side", 0), None, a.get("scale", 1.0), x, None, a.get("ws", x), a.get("bytes", big), None),
    }


@pytest.mark.parametrize("over,status,msg", BAD_QUANT)
def test_cache_descriptor_is_refused_everywhere(L, over, status, msg):
    for name, call in calls(L, c_quant(**over)).items():
        assert call() == status, name
        assert msg in L.prhs_last_error().decode(), name


def test_null_descriptor(L):
    x = 0x10000
    assert L.prhs_quant_store(None, x, x, 1, None, None, None) == B.PRHS_E_INVALID
    assert L.prhs_quant_dense_decode_attn(None, x, 1.0, x, None, x, 1 << 40, None) == B.PRHS_E_INVALID


@pytest.mark.parametrize("name,args,status", [
    ("store", dict(new_cap=-1), B.PRHS_E_INVALID),
    ("sparse", dict(cap=-1), B.PRHS_E_INVALID),
    ("sparse", dict(scale=float("nan")), B.PRHS_E_INVALID),
    ("dense", dict(ws=None), B.PRHS_E_WORKSPACE),
    ("dense", dict(bytes=16), B.PRHS_E_WORKSPACE),
    ("sparse", dict(bytes=16), B.PRHS_E_WORKSPACE),
    ("reuse", dict(anchor=None), B.PRHS_E_INVALID),
    ("pool", dict(rows=-1), B.PRHS_E_INVALID),
    ("pool", dict(side=5), B.PRHS_E_INVALID),
    ("pool", dict(side=1), B.PRHS_E_INVALID),
    ("pool", dict(unit=None), B.PRHS_E_INVALID),
])
def test_arguments_are_refused(L, name, args, status):
    assert calls(L, c_quant(), **args)[name]() == status
    assert L.prhs_last_error()


def test_store_refuses_bounds_that_do_not_fit(L):
    for bd, status in ((B.PrhsBounds(32, 0x100, 0x200), B.PRHS_E_INVALID),
                       (B.PrhsBounds(24, 0x100, 0x200), B.PRHS_E_UNSUPPORTED),
                       (B.PrhsBounds(16, None, 0x200), B.PRHS_E_INVALID),
                       (B.PrhsBounds(16, 0x100, 0x204), B.PRHS_E_INVALID)):
        assert calls(L, c_quant(), bd)["store"]() == status


def test_launches_beyond_the_grid_are_refused(L):
    # 2^31 / 16 tokens of rows in one store, and as many units' splits
    big = dict(batch=2048, num_q_heads=64, num_kv_heads=64, capacity=16000, max_seq_len=16000)
    assert calls(L, c_quant(**big), new_cap=16000)["store"]() == B.PRHS_E_UNSUPPORTED
    assert "workgroups" in L.prhs_last_error().decode()
    huge = dict(batch=1 << 19, num_q_heads=16, num_kv_heads=1, capacity=16, max_seq_len=16)
    assert calls(L, c_quant(**huge))["dense"]() == B.PRHS_E_UNSUPPORTED


def test_empty_batch_is_a_no_op(L):
    kv = c_quant(batch=0, k=None, v=None, seq_lens=None, k_scale=None, v_scale=None)
    r = ctypes.byref(kv)
    assert L.prhs_quant_store(r, None, None, 4, None, None, None) == B.PRHS_OK
    assert L.prhs_quant_dense_decode_attn(r, None, 1.0, None, None, None, 0, None) == B.PRHS_OK
    assert L.prhs_quant_sparse_decode_attn(r, None, None, None, 8, 1.0, None, None, None, 0, None) == B.PRHS_OK
    bd = B.PrhsBounds(16, None, None)
    assert L.prhs_block_bounds(ctypes.byref(kv.kv), ctypes.byref(bd), 1, None, None) == B.PRHS_OK
    p = B.params(k=16)
    assert L.prhs_block_select(ctypes.byref(kv.kv), None, ctypes.byref(p), ctypes.byref(bd), None, None,
                               1000, None, None, 1000, None, 0, None) == B.PRHS_OK


def test_max_blocks_and_set_capacity_hold_every_length(L):
    rng = random.Random(5)
    for _ in range(60):
        bs = rng.choice([16, 32, 64, 128])
        sink, window, s = rng.randrange(0, 200), rng.randrange(0, 300), rng.randrange(1, 9)
        kw = dict(k=rng.randrange(0, 900)) if rng.random() < 0.5 else dict(k_num=1, k_den=rng.randrange(1, 30))
        p = B.params(sink=sink, window=window, refresh_every=s, **kw)
        top = rng.randrange(0, 1500)
        most, cap = B.prhs_max_blocks(p, bs, top), B.prhs_block_set_capacity(p, bs, top)
        assert cap == min(top, sink + most * bs + window + s - 1)
        seen = 0
        for n in {0, 1, top, top // 2, max(0, top - 1), *(rng.randrange(0, top + 1) for _ in range(20))}:
            kb = n // p.k_den if p.k_den else p.k
            cand = Q.candidate_blocks(n, sink, window, bs)
            blocks = cand[: -(-kb // bs)]
            assert len(blocks) <= most
            assert len(Q.block_set(blocks, n, sink, window, bs)) <= min(top, sink + most * bs + window)
            if n == top:
                seen = len(blocks)
        assert seen == most
    for bad in ((p, 8, 100), (p, 16, -1), (B.params(k=-1), 16, 100)):
        assert B.prhs_max_blocks(*bad) == -1 and B.prhs_block_set_capacity(*bad) == -1
        assert L.prhs_last_error()


def c_select(L, kv, bd, p, **a):
    x = 0x10000
    return L.prhs_block_select(ctypes.byref(kv), a.get("q", x), ctypes.byref(p), ctypes.byref(bd), x, x,
                               a.get("blk_cap", 64), x, x, a.get("set_cap", 1000), a.get("ws", x),
                               a.get("bytes", 1 << 40), None)


@pytest.mark.parametrize("over,args,status,msg", [
    (dict(), dict(q=None), B.PRHS_E_INVALID, "non-NULL"),
    (dict(), dict(blk_cap=15), B.PRHS_E_CAPACITY, "blk_cap"),
    (dict(), dict(set_cap=4 + 256 + 63), B.PRHS_E_CAPACITY, "set_cap"),
    (dict(), dict(ws=None), B.PRHS_E_WORKSPACE, "workspace"),
    (dict(), dict(bytes=2 * 2 * 63 * 4 - 1), B.PRHS_E_WORKSPACE, "workspace"),
    (dict(seq_lens=None), dict(), B.PRHS_E_INVALID, "seq_lens"),
    (dict(capacity=1000), dict(), B.PRHS_E_INVALID, "capacity"),
])
def test_block_select_refusals(L, over, args, status, msg):
    p = B.params(k=256, sink=4, window=64)
    assert c_select(L, c_kv(**over), B.PrhsBounds(16, 0x100, 0x200), p, **args) == status
    assert msg in L.prhs_last_error().decode()


def test_block_select_takes_no_keys(L):
    # the refusal that ends this call comes after the cache's checks
    p = B.params(k=256, sink=4, window=64)
    assert c_select(L, c_kv(k=None, v=None), B.PrhsBounds(16, 0x100, 0x200), p, bytes=0) == B.PRHS_E_WORKSPACE
    n = ctypes.c_size_t(0)
    assert L.prhs_block_workspace_size(ctypes.byref(c_kv()), None, ctypes.byref(n)) == B.PRHS_E_INVALID


def test_attention_workspace_holds_every_smaller_call(L):
    rng = random.Random(9)

    def need(kv, dense, cap):
        st = calls(L, kv, cap=cap, bytes=0)["dense" if dense else "sparse"]()
        m = re.search(rb"workspace of (\d+) bytes", L.prhs_last_error())
        assert st == B.PRHS_E_WORKSPACE
        return int(m.group(1))

    for _ in range(60):
        hkv, g, d = rng.choice([1, 2, 8, 32]), rng.choice([1, 4, 16]), rng.choice([64, 128])
        batch, rows = rng.randrange(1, 80), 16 * rng.randrange(1, 2000)

        def kv(b, n):
            return c_quant(batch=b, num_q_heads=hkv * g, num_kv_heads=hkv, head_dim=d, capacity=rows, max_seq_len=n)

        for dense in (False, True):
            op = B.PRHS_OP_QUANT_DENSE_ATTN if dense else B.PRHS_OP_QUANT_SPARSE_ATTN
            n = ctypes.c_size_t(0)
            assert L.prhs_workspace_size(op, ctypes.byref(kv(batch, rows).kv), None, rows, ctypes.byref(n)) == B.PRHS_OK
            for b in {1, batch, (batch + 1) // 2, rng.randrange(1, batch + 1)}:
                for r in {1, rows, rng.randrange(1, rows + 1)}:
                    assert need(kv(b, r), dense, r) <= n.value, (batch, b, rows, r, hkv, g, d, dense)


# ---- the binding ----------------------------------------------------------------

def host_cache(paged=False, dtype=torch.bfloat16):
    e4 = torch.float8_e4m3fn
    n = torch.full((2,), 32, dtype=torch.int32)
    if paged:
        K = torch.zeros(6, 2, 16, 64, dtype=torch.uint8).view(e4)
        sc, table = torch.ones(6, 2), torch.zeros(2, 3, dtype=torch.int32)
        return B.QuantKV(K, K.clone(), sc, sc.clone(), n, 48, 8, table, dtype=dtype)
    K = torch.zeros(2, 2, 64, 64, dtype=torch.uint8).view(e4)
    return B.QuantKV(K, K.clone(), torch.ones(2, 2, 4), torch.ones(2, 2, 4), n, 64, 8, dtype=dtype)


def test_descriptors_of_the_binding():
    for paged in (False, True):
        kv = host_cache(paged)
        assert kv.block_size == 16 and kv.quant.block_size == 16 and kv.q_shape() == (2, 8, 64)
        lo = torch.zeros(6, 2, 64, dtype=kv.dtype) if paged else torch.zeros(2, 2, 4, 64, dtype=kv.dtype)
        assert B.BlockBounds(kv, lo, lo.clone()).block_size == 16
        with pytest.raises(ValueError):
            B.BlockBounds(kv, lo.float(), lo.float())
        with pytest.raises(ValueError):
            B.BlockBounds(kv, lo[..., :32].contiguous(), lo[..., :32].contiguous())
        assert kv.with_seq_lens(torch.zeros(2, dtype=torch.int32), 16).shape_c.max_seq_len == 16
    e4, n = torch.float8_e4m3fn, torch.zeros(2, dtype=torch.int32)
    K = torch.zeros(2, 2, 64, 64, dtype=torch.uint8).view(e4)
    for bad in (lambda: B.QuantKV(K.view(torch.uint8), K, torch.ones(2, 2, 4), torch.ones(2, 2, 4), n, 64, 8),
                lambda: B.QuantKV(K, K, torch.ones(2, 2, 3), torch.ones(2, 2, 3), n, 64, 8),
                lambda: B.QuantKV(K, K, torch.ones(2, 2, 4), torch.ones(2, 2, 2), n, 64, 8),
                lambda: B.QuantKV(K, K, torch.ones(2, 4), torch.ones(2, 4), n, 64, 8),
                lambda: B.QuantKV(K, K, torch.ones(2, 2, 4), torch.ones(2, 2, 4), n[:1], 64, 8),
                lambda: B.QuantKV(K, K, torch.ones(2, 2, 4), torch.ones(2, 2, 4), n, 64, 8, dtype=torch.float16),
                lambda: B.QuantKV(K, K[:, :1], torch.ones(2, 2, 4), torch.ones(2, 2, 4), n, 64, 8)):
        with pytest.raises(ValueError):
            bad()


def test_a_quantised_cache_is_refused_by_the_other_calls():
    kv = host_cache()
    q, out = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 8, 64)
    ws, i = torch.zeros(64, dtype=torch.uint8), torch.zeros(2, 2, 8, dtype=torch.int32)
    for call in (lambda: B.prhs_dense_decode_attn(kv, q, 1.0, out, None, ws),
                 lambda: B.prhs_sparse_decode_attn(kv, q, i, i[..., 0].contiguous(), 1.0, out, None, ws),
                 lambda: B.prhs_select(kv, q, B.params(k=4), i, i[..., 0].contiguous(), i, i[..., 0].contiguous(), ws),
                 lambda: B.prhs_prefill_attn(kv, torch.zeros(2, 8, 4, 64, dtype=torch.bfloat16), 1.0, torch.zeros(2, 8, 4, 64)),
                 lambda: B.prhs_block_bounds(kv, None, 1)):
        with pytest.raises(TypeError):
            call()
    K = torch.zeros(2, 2, 64, 64, dtype=torch.bfloat16)
    plain = B.KV(K, K, torch.zeros(2, dtype=torch.int32), 64, 8)
    with pytest.raises(TypeError):
        B.prhs_quant_dense_decode_attn(plain, q, 1.0, out, None, ws)
    with pytest.raises(TypeError):
        B.prhs_quant_store(plain, K, K)


def test_binding_refuses_shapes_and_host_tensors():
    kv = host_cache()
    bf, i32 = torch.bfloat16, torch.int32
    q, out, lse = torch.zeros(2, 8, 64, dtype=bf), torch.zeros(2, 8, 64), torch.zeros(2, 8)
    ws, sets, lens = torch.zeros(64, dtype=torch.uint8), torch.zeros(2, 2, 40, dtype=i32), torch.zeros(2, 2, dtype=i32)
    new = torch.zeros(2, 2, 3, 64, dtype=bf)
    bd = B.BlockBounds(kv, torch.zeros(2, 2, 4, 64, dtype=bf), torch.zeros(2, 2, 4, 64, dtype=bf))
    other = B.BlockBounds(host_cache(True), torch.zeros(6, 2, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf))
    bad = [
        lambda: B.prhs_quant_store(kv, new, new[:, :, :2].contiguous()),
        lambda: B.prhs_quant_store(kv, new.float(), new.float()),
        lambda: B.prhs_quant_store(kv, new[:, :, :, :32].contiguous(), new[:, :, :, :32].contiguous()),
        lambda: B.prhs_quant_store(kv, new.transpose(1, 2), new.transpose(1, 2)),
        lambda: B.prhs_quant_store(kv, new, new, torch.zeros(3, dtype=i32)),
        lambda: B.prhs_quant_store(kv, new, new, None, other),
        lambda: B.prhs_quant_dense_decode_attn(kv, q.float(), 1.0, out, lse, ws),
        lambda: B.prhs_quant_dense_decode_attn(kv, q, 1.0, out[:1], lse, ws),
        lambda: B.prhs_quant_sparse_decode_attn(kv, q, sets, lens[:1], 1.0, out, lse, ws),
        lambda: B.prhs_quant_reuse_decode_attn(kv, q, sets, lens, torch.zeros(3, dtype=i32), 1.0, out, lse, ws),
        lambda: B.prhs_quant_pool_decode_attn(kv, q, sets, lens, torch.zeros(3, dtype=i32), torch.zeros(4, dtype=i32), 1.0, out, lse, ws),
        lambda: B.prhs_block_select(kv, q, B.params(k=4), other, sets, lens, sets, lens, ws),
        lambda: B.prhs_block_select(kv, q, B.params(k=4), bd, sets, lens[:1], sets, lens, ws),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"case {i} was not refused")
    host = [
        lambda: B.prhs_quant_store(kv, new, new, None, bd),
        lambda: B.prhs_quant_dense_decode_attn(kv, q, 1.0, out, lse, ws),
        lambda: B.prhs_quant_sparse_decode_attn(kv, q, sets, lens, 1.0, out, lse, ws),
        lambda: B.prhs_block_select(kv, q, B.params(k=4), bd, sets, lens, sets, lens, ws),
    ]
    for call in host:
        with pytest.raises(ValueError, match="GPU"):
            call()
