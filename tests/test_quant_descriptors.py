"""Descriptors of the 8-bit cache on the host: scales of another rank, and the
workspace of a cache with many rows."""

import ctypes

import pytest
import torch

from paper_2602_08329_amd import binding as B

E4 = torch.float8_e4m3fn


@pytest.mark.parametrize("paged", [False, True])
def test_scales_have_one_entry_a_block_and_head(paged):
    n = torch.zeros(2, dtype=torch.int32)
    K = torch.zeros((6, 2, 16, 64) if paged else (2, 2, 64, 64), dtype=torch.uint8).view(E4)
    table = torch.zeros(2, 3, dtype=torch.int32) if paged else None
    good = (6, 2) if paged else (2, 2, 4)

    def make(*shape):
        return B.QuantKV(K, K, torch.ones(shape), torch.ones(shape), n, 48, 8, table)

    assert make(*good).block_size == 16
    for shape in (good + (5,), good + (1,), good[:-1], (1,) + good):
        with pytest.raises(ValueError, match="k_scale"):
            make(*shape)


def test_block_workspace_of_many_rows():
    # 2^32 rows of one block, whose keys are kept in eights
    c = B.PrhsKv(1 << 20, 4096, 4096, 64, B.PRHS_BF16, B.PRHS_KV_PAGED, 0, 16, 1, 8, None, None, None, None, 16)
    b, n = B.PrhsBounds(16, None, None), ctypes.c_size_t(0)
    assert B.lib().prhs_block_workspace_size(ctypes.byref(c), ctypes.byref(b), ctypes.byref(n)) == B.PRHS_OK
    assert n.value == 2 ** 32 * 8 * 4
