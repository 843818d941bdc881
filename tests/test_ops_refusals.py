"""Calls of the cache operators that are refused before anything reaches a device (CPU only)."""
from __future__ import annotations

import ctypes
import math
import os

import pytest
import torch

from paper_2608_28099_amd import binding, ops
from tests.test_ops_cpu import P, UNSUPPORTED, rows, store

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


def test_scales_that_fp32_does_not_hold():
    """A positive scale that fp32 rounds to 0 would ask for the default one."""
    k = torch.zeros(4, 2, 2048, dtype=torch.bfloat16)
    cache = ops.PagedCache(k, k, 16, torch.zeros(1, 2, dtype=torch.int32))
    x = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16)
    for scale in (1e-46, 1e-60, 1e39, 1e300, 0.0, -0.5, math.inf, math.nan):
        with pytest.raises(ValueError, match="scale"):
            ops.tree_attention(cache, torch.zeros(1, dtype=torch.int32), x, x, x, scale=scale)
    cfg = binding.sp_tree_config(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=1, kv_dtype=1, max_nodes=8, max_batch=2,
                                 max_seq_len=64)
    largest = 3.4028234663852886e38
    for scale, good in ((1e-40, True), (0.69 * largest, True), (0.7 * largest, False), (largest, False)):
        cfg.scale = scale                                 # (times log2(e) it has to be finite too)
        assert (binding.load().sp_probe_tree_workspace_bytes(ctypes.byref(cfg)) > 0) == good, scale


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_frequencies_that_the_scaling_does_not_use(scaling):
    kw = dict(scaling=scaling, factor=2.0, original_positions=4096)
    ops.make_rotary(64, **kw)
    with pytest.raises(ValueError, match="frequencies"):
        ops.make_rotary(64, frequencies=[0.5] * 32, **kw)


@pytest.mark.parametrize("dtype,element", [(binding.SP_F32, 4), (binding.SP_BF16, 2), (binding.SP_E4M3, 1)])
@pytest.mark.parametrize("hd", [64, 128])
def test_blocks_past_the_offsets_within_them(dtype, element, hd):
    """A head's block of more than 2^31 bytes; the largest that is taken gets past this check, to one of the workspace."""
    most = (1 << 31) // (hd * element)
    cfg = binding.sp_tree_config(n_q_heads=8, n_kv_heads=2, head_dim=hd, dtype=min(dtype, 1), kv_dtype=dtype, max_nodes=8,
                                 max_batch=2, max_seq_len=64)
    t = binding.sp_tree(n_nodes=4, q=rows(8), k=rows(2), v=rows(2), out=rows(8))
    for block, want in ((2 * most, UNSUPPORTED), (4 * most, UNSUPPORTED), (most, -1), (16, -1)):
        head = block * hd
        kw = dict(exponent_stride_block=2 * block, exponent_stride_head=block) if element == 1 else {}
        s = store(dtype, head_dim=hd, block_size=block, k_stride_head=head, v_stride_head=head, k_stride_block=2 * head,
                  v_stride_block=2 * head, **kw)
        assert binding.load().sp_probe_tree_attention(ctypes.byref(cfg), ctypes.byref(s), P, P, ctypes.byref(t), P, 0, None) == want


def test_workspaces_of_other_types():
    k = torch.zeros(4, 2, 2048, dtype=torch.bfloat16)
    cache = ops.PagedCache(k, k, 16, torch.zeros(1, 2, dtype=torch.int32))
    assert ops.tree_workspace_bytes(cache, 8, torch.bfloat16, 4) > 0
    assert ops.tree_workspace_bytes(cache, 8, torch.float32, 4) == 0          # of a bf16 cache: not supported
    for dtype in (torch.float16, torch.float8_e4m3fn, None):
        with pytest.raises(ValueError):
            ops.tree_workspace_bytes(cache, 8, dtype, 4)
