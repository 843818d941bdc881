"""Calls of the cache operators that are refused before anything reaches a device (CPU only)."""
from __future__ import annotations

import os

import pytest
import torch

from paper_2608_28099_amd import binding, ops

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH),
                                reason="libsp_probe.so not built (run __graft_entry__.build())")


def test_rows_of_a_batch_of_trees():
    """[batch, nodes, heads, head_dim] is what tree attention takes; rotations, writing and reading take rows."""
    k = torch.zeros(4, 2, 2048, dtype=torch.bfloat16)
    cache = ops.PagedCache(k, k, 16, torch.zeros(2, 2, dtype=torch.int32))
    x, flat = torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16), torch.zeros(2, 2, 128, dtype=torch.bfloat16)
    ids, rot = torch.zeros(2, dtype=torch.int32), ops.make_rotary(128)
    shape = r"must be \[rows, heads"
    for call in (lambda: ops.rotary(rot, ids, x), lambda: ops.rotary(rot, ids, flat, x), lambda: ops.rotary(rot, ids, x, out=x),
                 lambda: ops.rotary(rot, ids, x, x), lambda: ops.cache_write(cache, ids, ids, x, x),
                 lambda: ops.cache_write(cache, ids, ids, flat, x), lambda: ops.cache_read(cache, ids, ids, k=x, v=x),
                 lambda: ops.cache_read(cache, ids, ids, v=x), lambda: ops.cache_read(cache, ids, ids, k=x, v=flat)):
        with pytest.raises(ValueError, match=shape):
            call()
