"""Which calls of the 8-bit cache are too large to launch: those of 2^32 threads
or more, counted as the launch counts them.  Every call here ends in a refusal,
of its size or of an argument that is checked after it."""

import ctypes

import pytest

from paper_2602_08329_amd import binding as B


@pytest.fixture(scope="module")
def L():
    return B.lib()


def kv(**over):
    f = dict(batch=64, num_q_heads=32, num_kv_heads=32, head_dim=128, dtype=B.PRHS_BF16,
             layout=B.PRHS_KV_CONTIGUOUS, capacity=32768, page_size=16, max_pages=64, num_pages=128,
             k=0x1000, v=0x2000, block_table=0x9000, seq_lens=0x3000, max_seq_len=32768)
    f.update(over)
    return B.PrhsKv(**f)


def store(L, c, bs, new_cap):
    q = B.PrhsQuantKv(c, bs, 0x5000, 0x6000)
    return L.prhs_quant_store(ctypes.byref(q), None, None, new_cap, None, None, None)


@pytest.mark.parametrize("over,bs,new_cap", [
    (dict(), 16, 32768),                                # 64 prompts of 32k: 2 x 2^20 workgroups
    (dict(), 128, 32768),
    (dict(head_dim=64), 16, 32768),
    (dict(batch=1 << 17, capacity=16, max_seq_len=16), 16, 1),      # many short ones
])
def test_large_stores_are_taken(L, over, bs, new_cap):
    assert store(L, kv(**over), bs, new_cap) == B.PRHS_E_INVALID
    assert "k_new" in L.prhs_last_error().decode()


def test_stores_of_too_many_threads_are_refused(L):
    # blocks of 16 tokens: four a workgroup of 256 threads, K and V apart, so that
    # 2^25 blocks are 2^32 threads; a prompt of whole blocks touches all of them
    def blocks(n, bs=16):
        return kv(batch=n, num_q_heads=32, num_kv_heads=32, capacity=bs, max_seq_len=bs)

    assert store(L, blocks((1 << 20) - 1), 16, 16) == B.PRHS_E_INVALID
    assert store(L, blocks(1 << 20), 16, 16) == B.PRHS_E_UNSUPPORTED
    assert "workgroups" in L.prhs_last_error().decode()
    # of 128 tokens: one
    assert store(L, blocks((1 << 18) - 1, 128), 128, 128) == B.PRHS_E_INVALID
    assert store(L, blocks(1 << 18, 128), 128, 128) == B.PRHS_E_UNSUPPORTED


def test_bounds_of_too_many_threads_are_refused(L):
    # 2^26 blocks of 16 tokens, four a workgroup
    c = kv(batch=1 << 21, layout=B.PRHS_KV_PAGED, max_pages=1, num_pages=64, max_seq_len=16)
    b = B.PrhsBounds(16, 0x100, 0x200)
    assert L.prhs_block_bounds(ctypes.byref(c), ctypes.byref(b), 16, None, None) == B.PRHS_E_UNSUPPORTED
    assert "workgroups" in L.prhs_last_error().decode()


def select(L, c, bs):
    p, b = B.params(k=bs), B.PrhsBounds(bs, 0x100, 0x200)
    return L.prhs_block_select(ctypes.byref(c), 0x100, ctypes.byref(p), ctypes.byref(b), 0x100, 0x100, 1 << 20,
                               0x100, 0x100, 1 << 22, None, 0, None)


@pytest.mark.parametrize("over,bs", [
    (dict(batch=256, num_q_heads=32, num_kv_heads=32, capacity=131072, max_seq_len=131072), 16),
    (dict(batch=1 << 17, capacity=256, max_seq_len=256), 16),
    (dict(batch=1 << 17, dtype=B.PRHS_F32, layout=B.PRHS_KV_PAGED, max_pages=2, max_seq_len=32), 16),
])
def test_large_selections_are_taken(L, over, bs):
    assert select(L, kv(**over), bs) == B.PRHS_E_WORKSPACE


def test_selections_of_too_many_threads_are_refused(L):
    # one workgroup of 512 threads a row
    c = dict(layout=B.PRHS_KV_PAGED, max_pages=1, num_pages=64, max_seq_len=16)
    assert select(L, kv(batch=(1 << 18) - 1, **c), 16) == B.PRHS_E_WORKSPACE
    assert select(L, kv(batch=1 << 18, **c), 16) == B.PRHS_E_UNSUPPORTED
