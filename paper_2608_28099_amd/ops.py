"""Operators on a speculative head's paged cache, for torch tensors.

    rot = ops.make_rotary(128, scaling="yarn", factor=4.0, original_positions=32768)
    q, k = ops.rotary(rot, positions, q, k)                     # rotate projections
    ops.cache_write(cache, seq_ids, positions, k, v)            # put them into the cache
    out = ops.tree_attention(cache, seq_lens, q, k, v, mask)    # a drafted tree over it
    k, v = ops.cache_read(cache, seq_ids, positions, torch.bfloat16)

Thin marshalling over the C functions of include/sp_probe.h (sp_probe_rotary,
sp_probe_cache_write, sp_probe_cache_read, sp_probe_tree_attention), which document the
operations.  Calls go to the given stream (a raw handle; default: the current
stream of the tensors' device) and return without waiting; a given stream's order against the
streams that made the inputs and read the results is the caller's to keep.  Wrong types, shapes and
devices raise ValueError here, what the library refuses raises binding.ProbeError.
Results carry no autograd graph: a rotation's gradient is its transpose, and the other operators are
for serving.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding
from .binding import ProbeError, SP_BF16, SP_E4M3, SP_F32, SP_OK

_ROW_TYPES = {torch.float32: SP_F32, torch.bfloat16: SP_BF16}
_CACHE_TYPES = {torch.float32: SP_F32, torch.bfloat16: SP_BF16, torch.float8_e4m3fn: SP_E4M3}
_MASK_TYPES = (torch.int32, torch.uint32)
_LAYOUTS = {"half": binding.SP_ROTARY_HALF, "interleaved": binding.SP_ROTARY_INTERLEAVED}
_SCALINGS = {"none": binding.SP_ROTARY_PLAIN, "linear": binding.SP_ROTARY_LINEAR, "ntk": binding.SP_ROTARY_NTK,
             "yarn": binding.SP_ROTARY_YARN, "custom": binding.SP_ROTARY_CUSTOM}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


# Every call runs with its tensors' device current (else it calls itself under a guard) and on
# the raw handle of the given or current stream.  The checks of a call spell out what is wrong
# only where they fail: a call's host time is of the order of its kernel's.
_current_device = torch.cuda.current_device
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _elsewhere(device):
    """Whether `device` is not the current one."""
    if device.type != "cuda":
        raise ValueError("tensors must be on the GPU")
    return device.index is not None and device.index != _current_device()


def _empty(shape, dtype, device, stream):
    """Memory for a call: of the given stream's pool, so that nothing enqueued elsewhere still uses it, and
    once freed not handed out again before the current stream, which may read it, is past that."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    now = torch.cuda.current_stream(device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(now)
    return t


def _empty_like(t, stream):
    if stream is None:  # (half the host time of torch.empty)
        return torch.empty_like(t, memory_format=torch.contiguous_format)
    return _empty(t.shape, t.dtype, t.device, stream)


def _check(status, what):
    if status != SP_OK:
        raise ProbeError(status, what)


def _rows(t, name, head_dim, dtype, device, n=None):
    """sp_rows of a [rows, heads, head_dim] tensor, or [batch, nodes, heads, head_dim] with evenly spaced rows."""
    shape, stride = t.shape, t.stride()
    if not 3 <= len(shape) <= 4 or shape[-1] != head_dim:
        raise ValueError(f"{name} must be [rows, heads, {head_dim}]")
    if t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be {dtype} on {device}")
    if stride[-1] != 1:
        raise ValueError(f"{name}: the values of a head must lie side by side")
    row = stride[-3]
    if len(shape) == 4 and shape[0] != 1:
        if shape[1] == 1:
            row = stride[0]  # (the stride of a dimension of one means nothing)
        elif stride[0] != shape[1] * row:
            raise ValueError(f"{name}: rows must be evenly spaced")
    if n is not None and shape[0] != n:
        raise ValueError(f"{name} must have {n} rows")
    return binding.sp_rows(t.data_ptr(), row, stride[-2], shape[-2], 0)


def _ids(t, name, n, device):
    if t.dtype != torch.int32 or t.device != device or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be {n} contiguous int32 on {device}")
    return t.data_ptr()


# ---------------------------------------------------------------- rotary

def make_rotary(head_dim, rotary_dim=None, base=10000.0, layout="half", scaling="none", factor=1.0,
                original_positions=0, beta_fast=0.0, beta_slow=0.0, attn_factor=0.0, frequencies=None):
    """The rotation (a binding.sp_rotary, host data) of the first rotary_dim values of a head.
    scaling: "none", "linear", "ntk", "yarn", or "custom" with frequencies (radians per position)."""
    _need(layout in _LAYOUTS, f"layout must be one of {sorted(_LAYOUTS)}")
    _need(scaling in _SCALINGS, f"scaling must be one of {sorted(_SCALINGS)}")
    dim = head_dim if rotary_dim is None else rotary_dim
    cfg = binding.sp_rotary_config(head_dim=head_dim, rotary_dim=dim, layout=_LAYOUTS[layout],
                                   scaling=_SCALINGS[scaling], base=base, factor=factor,
                                   original_positions=original_positions, beta_fast=beta_fast, beta_slow=beta_slow,
                                   attn_factor=attn_factor)
    _need(frequencies is None or scaling == "custom", 'frequencies go with scaling="custom" alone')
    if frequencies is not None:
        f = [float(x) for x in frequencies]
        _need(len(f) == dim // 2, f"frequencies must hold {dim // 2} values")
        cfg.frequencies = (ctypes.c_double * len(f))(*f)
    out = binding.sp_rotary()
    _check(binding.load().sp_probe_rotary_init(ctypes.byref(cfg), ctypes.byref(out)), "sp_probe_rotary_init")
    return out


def rotary(rot, positions, q, k=None, out=None, k_out=None, transpose=False, stream=None):
    """q [rows, heads, head_dim] (and k) rotated at positions (int32 [rows]): returns the
    rotated q, or (q, k).  out, k_out: where to write (the inputs themselves: in place);
    rows at negative positions are not written.  transpose: the gradient's rotation (by
    the opposite angle, with the same factor)."""
    hd, dev, dtype, n = rot.head_dim, q.device, q.dtype, q.shape[0]
    if dtype not in _ROW_TYPES:
        raise ValueError("q must be float32 or bfloat16")
    if q.dim() != 3 or (k is not None and k.dim() != 3):  # (_rows knows the nodes of a batch too)
        raise ValueError("q and k must be [rows, heads, head_dim]")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return rotary(rot, positions, q, k, out, k_out, transpose, stream)
    if out is None:
        out = _empty_like(q, stream)
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    qr, outr = _rows(q, "q", hd, dtype, dev, n), _rows(out, "out", hd, dtype, dev, n)
    kr = k_outr = None
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    if k is not None:
        if k_out is None:
            k_out = _empty_like(k, stream)
        elif k_out.shape != k.shape:
            raise ValueError("k_out must have k's shape")
        kr, k_outr = _rows(k, "k", hd, dtype, dev, n), _rows(k_out, "k_out", hd, dtype, dev, n)
    _check(binding.load().sp_probe_rotary(rot, _ROW_TYPES[dtype], 1 if transpose else 0, n,
                                          _ids(positions, "positions", n, dev), qr, outr, kr, k_outr,
                                          _current_stream(_current_device()) if stream is None else stream),
           "sp_probe_rotary")
    return out if k is None else (out, k_out)


# ---------------------------------------------------------------- the paged cache

class PagedCache:
    """A paged cache: keys and values [num_blocks, n_kv_heads, block_size * head_dim] in the
    layout of include/sp_probe.h (float32, bfloat16, or float8_e4m3fn with uint8 exponents
    [num_blocks, n_kv_heads, block_size]).  block_table int32 [batch, blocks]; without one, storage
    is contiguous and batch says how many sequences share the blocks evenly."""

    def __init__(self, k, v, block_size, block_table=None, k_exponents=None, v_exponents=None, batch=None):
        _need(k.dtype in _CACHE_TYPES and v.dtype == k.dtype, "k and v must both be float32, bfloat16 or float8_e4m3fn")
        _need(k.dim() == 3 and v.shape == k.shape and v.device == k.device, "k and v must be [blocks, heads, block_size * head_dim]")
        _need(k.stride(-1) == 1 and v.stride(-1) == 1, "a head's block must be contiguous")
        _need(block_size > 0 and k.shape[2] % block_size == 0, "the last dimension must hold block_size * head_dim values")
        self.k, self.v, self.block_size, self.block_table = k, v, block_size, block_table
        self.k_exponents, self.v_exponents = k_exponents, v_exponents
        self.num_blocks, self.n_kv_heads = k.shape[0], k.shape[1]
        self.head_dim, self.dtype, self.device = k.shape[2] // block_size, k.dtype, k.device
        if block_table is not None:
            _need(block_table.dtype == torch.int32 and block_table.dim() == 2 and block_table.is_contiguous()
                  and block_table.device == k.device, "block_table must be contiguous int32 [batch, blocks] beside k")
            self.batch, self.max_blocks = block_table.shape
            _need(batch is None or batch == self.batch, "batch must be the block table's")
        else:
            _need(batch is not None and batch > 0 and self.num_blocks >= batch, "contiguous storage needs batch")
            self.batch, self.max_blocks = batch, self.num_blocks // batch
        st = binding.sp_kv_store(dtype=_CACHE_TYPES[k.dtype], n_kv_heads=self.n_kv_heads, head_dim=self.head_dim)
        st.kv = binding.sp_kv_cache(k_base=k.data_ptr(), v_base=v.data_ptr(), num_blocks=self.num_blocks,
                                    k_stride_block=k.stride(0), k_stride_head=k.stride(1),
                                    v_stride_block=v.stride(0), v_stride_head=v.stride(1),
                                    block_size=block_size, max_blocks_per_seq=self.max_blocks, batch=self.batch)
        if k.dtype == torch.float8_e4m3fn:
            for e in (k_exponents, v_exponents):
                _need(e is not None and e.dtype == torch.uint8 and e.device == k.device and e.stride(-1) == 1
                      and tuple(e.shape) == (self.num_blocks, self.n_kv_heads, block_size),
                      "float8 caches need uint8 exponents [blocks, heads, block_size]")
            _need(k_exponents.stride() == v_exponents.stride(), "both exponents must have the same strides")
            st.k_exponents, st.v_exponents = k_exponents.data_ptr(), v_exponents.data_ptr()
            st.exponent_stride_block, st.exponent_stride_head = k_exponents.stride(0), k_exponents.stride(1)
        else:
            _need(k_exponents is None and v_exponents is None, "exponents belong to float8 caches")
        self.c, self.c_dtype = st, st.dtype
        self.table = None if block_table is None else block_table.data_ptr()
        self.capacity = min(self.max_blocks * block_size, 1 << 30)  # tokens of a sequence that attention reads

    @classmethod
    def allocate(cls, dtype, num_blocks, n_kv_heads, head_dim, block_size=16, block_table=None, batch=None, device="cuda"):
        """A zeroed cache: one pool [num_blocks, n_kv_heads, 2, block_size * head_dim]."""
        pool = torch.zeros((num_blocks, n_kv_heads, 2, block_size * head_dim), dtype=dtype, device=device)
        e = None
        if dtype == torch.float8_e4m3fn:
            e = torch.full((num_blocks, n_kv_heads, 2, block_size), 127, dtype=torch.uint8, device=device)
        return cls(pool[:, :, 0], pool[:, :, 1], block_size, block_table, None if e is None else e[:, :, 0],
                   None if e is None else e[:, :, 1], batch)

    @classmethod
    def from_kv(cls, kv):
        """The cache of an inputs.KVCache (what Probe.forward reads), sharing its memory."""
        return cls(kv.pool[:, :, 0], kv.pool[:, :, 1], kv.block_size, kv.block_table,
                   batch=None if kv.block_table is not None else kv.seq_lens.shape[0])


def cache_write(cache: PagedCache, seq_ids, positions, k, v, src_rows=None, rotary=None, stream=None):
    """Row i of k and v (row src_rows[i]; all [rows, n_kv_heads, head_dim], float32 or bfloat16)
    becomes token positions[i] of sequence seq_ids[i]; the key is rotated there first if a
    rotation is given.  Rows with ids or positions out of range are skipped; the slots of a
    call must differ."""
    dev, n, dtype, hd = cache.device, seq_ids.shape[0], k.dtype, cache.head_dim
    if dtype not in _ROW_TYPES or k.dim() != 3 or v.dim() != 3:
        raise ValueError("k and v must be [rows, heads, head_dim], float32 or bfloat16")
    n_src = k.shape[0]
    if src_rows is None and n_src != n:
        raise ValueError(f"k must have {n} rows")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return cache_write(cache, seq_ids, positions, k, v, src_rows, rotary, stream)
    _check(binding.load().sp_probe_cache_write(
        cache.c, cache.table, _ROW_TYPES[dtype], n, _ids(seq_ids, "seq_ids", n, dev),
        _ids(positions, "positions", n, dev), None if src_rows is None else _ids(src_rows, "src_rows", n, dev),
        n_src, _rows(k, "k", hd, dtype, dev), _rows(v, "v", hd, dtype, dev, n_src), rotary,
        _current_stream(_current_device()) if stream is None else stream), "sp_probe_cache_write")


def cache_read(cache: PagedCache, seq_ids, positions, dtype=torch.bfloat16, k=None, v=None, stream=None):
    """Tokens positions[i] of sequences seq_ids[i] as rows [rows, n_kv_heads, head_dim] (k, v) of
    dtype; given k and v (either or both) are written instead: rows with ids or positions out
    of range are left as they are."""
    dev, n, hd = cache.device, seq_ids.shape[0], cache.head_dim
    if (k is not None and k.dim() != 3) or (v is not None and v.dim() != 3):
        raise ValueError("k and v must be [rows, heads, head_dim]")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return cache_read(cache, seq_ids, positions, dtype, k, v, stream)
    if k is None and v is None:
        k = _empty((n, cache.n_kv_heads, hd), dtype, dev, stream)
        v = _empty_like(k, stream)
    else:
        dtype = k.dtype if k is not None else v.dtype
    if dtype not in _ROW_TYPES:
        raise ValueError("rows must be float32 or bfloat16")
    _check(binding.load().sp_probe_cache_read(
        cache.c, cache.table, _ROW_TYPES[dtype], n, _ids(seq_ids, "seq_ids", n, dev),
        _ids(positions, "positions", n, dev), None if k is None else _rows(k, "k", hd, dtype, dev, n),
        None if v is None else _rows(v, "v", hd, dtype, dev, n),
        _current_stream(_current_device()) if stream is None else stream), "sp_probe_cache_read")
    return k, v


# ---------------------------------------------------------------- tree attention

def tree_mask(parents):
    """The mask words (int32 [.., nodes, ceil(nodes / 32)]) of trees given by parents (integers
    [.., nodes], -1 at a root, each before its children): a node sees itself and its ancestors."""
    parents = torch.as_tensor(parents)
    t = parents.shape[-1]
    flat = parents.reshape(-1, t).cpu().tolist()
    words = torch.zeros((len(flat), t, -(-t // 32)), dtype=torch.int64)
    for b, row in enumerate(flat):
        for i, at in enumerate(row):
            _need(-1 <= at < i, "a parent comes before its children")
            if at >= 0:
                words[b, i] = words[b, at]
            words[b, i, i // 32] |= 1 << (i % 32)
    words = torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)
    return words.reshape(*parents.shape, -1).to(parents.device)


def _tree_config(cache, n_q_heads, dtype, nodes, batch, max_seq_len, scale):
    return binding.sp_tree_config(n_q_heads, cache.n_kv_heads, cache.head_dim, _ROW_TYPES[dtype], cache.c_dtype, nodes,
                                  batch, max_seq_len, scale, 0)


def tree_attention(cache: PagedCache, seq_lens, q, k, v, mask=None, counts=None, max_seq_len: Optional[int] = None,
                   scale: Optional[float] = None, out=None, lse=None, workspace=None, stream=None):
    """Attention of the nodes q [batch, nodes, n_q_heads, head_dim] over the seq_lens (int32
    [batch]) cached tokens of each sequence and the nodes' own keys and values k, v
    [batch, nodes, n_kv_heads, head_dim] as mask shows them: int32 words [batch, nodes, words]
    or [nodes, words] (tree_mask; bit j of word w of node i: it sees node 32 w + j); None: each
    node sees those up to itself.  counts (int32 [batch]): nodes of each sequence; rows past
    them are not written.  max_seq_len: the longest sequence, which plans the launch (default:
    what the block table holds).  lse: float32 [batch, nodes, n_q_heads] to
    receive ln sum exp(score).  workspace: a uint8 tensor to use instead of fresh memory."""
    dev, hd, dtype, shape = cache.device, cache.head_dim, q.dtype, q.shape
    if dtype not in _ROW_TYPES:
        raise ValueError("q must be float32 or bfloat16")
    if len(shape) != 4 or k.dim() != 4 or v.shape != k.shape or k.shape[:2] != shape[:2]:
        raise ValueError("q, k and v must be [batch, nodes, heads, head_dim]")
    batch, nodes, nq = shape[:3]
    if batch != cache.batch:
        raise ValueError(f"the cache has {cache.batch} sequences")
    if k.shape[2] != cache.n_kv_heads:
        raise ValueError(f"the cache has {cache.n_kv_heads} KV heads")
    if max_seq_len is None:
        max_seq_len = cache.capacity
    if scale is None:
        scale = 0.0
    else:
        scale = ctypes.c_float(scale).value  # what the library receives; its 0 means the default
        if not (math.isfinite(scale) and scale > 0):
            raise ValueError("scale must be positive and within float32's range")
    if _elsewhere(dev):
        with torch.cuda.device(dev):
            return tree_attention(cache, seq_lens, q, k, v, mask, counts, max_seq_len, scale or None, out, lse, workspace,
                                  stream)
    if out is None:
        out = _empty_like(q, stream)
    elif out.shape != shape:
        raise ValueError("out must have q's shape")
    tree = binding.sp_tree(nodes, 0, None if counts is None else _ids(counts, "counts", batch, dev), None, 0,
                           _rows(q, "q", hd, dtype, dev), _rows(k, "k", hd, dtype, dev),
                           _rows(v, "v", hd, dtype, dev), _rows(out, "out", hd, dtype, dev), None)
    if mask is not None:
        words = mask.shape
        if (mask.dtype not in _MASK_TYPES or mask.device != dev or not mask.is_contiguous()
                or not 2 <= len(words) <= 3 or words[-2] != nodes or (len(words) == 3 and words[0] != batch)):
            raise ValueError("mask must be contiguous int32 words [batch, nodes, words] or [nodes, words]")
        tree.mask, tree.mask_words = mask.data_ptr(), words[-1]
        tree.mask_stride = 0 if len(words) == 2 else nodes * words[-1]
    if lse is not None:
        if lse.dtype != torch.float32 or lse.device != dev or not lse.is_contiguous() or lse.shape != shape[:3]:
            raise ValueError("lse must be contiguous float32 [batch, nodes, n_q_heads]")
        tree.lse = lse.data_ptr()
    cfg = _tree_config(cache, nq, dtype, nodes, batch or 1, max_seq_len, scale)
    lib = binding.load()
    if workspace is None:
        workspace = _empty(max(lib.sp_probe_tree_workspace_bytes(cfg), 16), torch.uint8, dev, stream)
    elif workspace.dtype != torch.uint8 or workspace.device != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be contiguous uint8 on {dev}")
    _check(lib.sp_probe_tree_attention(cfg, cache.c, _ids(seq_lens, "seq_lens", batch, dev), cache.table, tree,
                                       workspace.data_ptr(), workspace.numel(),
                                       _current_stream(_current_device()) if stream is None else stream),
           "sp_probe_tree_attention")
    return out


def tree_workspace_bytes(cache: PagedCache, n_q_heads, dtype, nodes, batch=None, max_seq_len=None):
    """Bytes of workspace that tree_attention needs for calls of at most these nodes, with this batch and
    max_seq_len, which plan the launch (0: not supported)."""
    if dtype not in _ROW_TYPES:
        raise ValueError("dtype must be float32 or bfloat16")
    if cache.device.type == "cuda" and _elsewhere(cache.device):  # the launch is planned for its compute units
        with torch.cuda.device(cache.device):
            return tree_workspace_bytes(cache, n_q_heads, dtype, nodes, batch, max_seq_len)
    return binding.load().sp_probe_tree_workspace_bytes(
        _tree_config(cache, n_q_heads, dtype, nodes, cache.batch if batch is None else batch,
                     cache.capacity if max_seq_len is None else max_seq_len, 0.0))
