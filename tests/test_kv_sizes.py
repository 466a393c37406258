"""Sizes of the cache's binding that pass 32 bits are refused, not cut."""
from __future__ import annotations

import pytest
import torch

from paper_2606_11244_amd import kv


def _cache():
    return kv.Cache(torch.zeros(3, 2, 16, 64, dtype=torch.int8), torch.zeros(3, 2, 64, 16, dtype=torch.int8), torch.ones(3, 2),
                    torch.ones(3, 2), torch.float16)


@pytest.mark.parametrize("far", [2 ** 31, 2 ** 32 + 1, 2 ** 63 - 1, -2 ** 31 - 1])
def test_sizes_past_32_bits(far):
    table = torch.zeros(4, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="32 bits"):
        kv.Batch(table, far)
    with pytest.raises(ValueError, match="32 bits"):
        kv.Batch(table, 5, max_new=far)
    batch = kv.Batch(table, 5)
    with pytest.raises(ValueError, match="32 bits"):
        kv.AttentionPlan(_cache(), batch, 2, window=far)
    with pytest.raises(ValueError, match="32 bits"):
        kv.AttentionPlan(_cache(), batch, far)


def test_a_tables_stride_past_32_bits():
    far = torch.empty(1, dtype=torch.int32, device="meta").as_strided((2, 4), (2 ** 32 + 4, 1))
    with pytest.raises(ValueError, match="32 bits"):
        kv.Batch(far, 5)


def test_sizes_of_32_bits_go_to_the_library():
    table = torch.zeros(4, 8, dtype=torch.int32)
    assert kv.AttentionPlan(_cache(), kv.Batch(table, 5), 2, window=2 ** 31 - 1).c.window == 2 ** 31 - 1
    with pytest.raises(kv.SpearError):
        kv.AttentionPlan(_cache(), kv.Batch(table, 5), 2, window=-1)
    with pytest.raises(kv.SpearError):
        kv.AttentionPlan(_cache(), kv.Batch(table, 5, max_new=-2 ** 31), 2)
