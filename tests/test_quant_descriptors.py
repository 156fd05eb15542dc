"""Descriptors of the 8-bit cache on the host: scales of another rank."""

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
