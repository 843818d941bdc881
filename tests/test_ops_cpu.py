"""The cache operators' host side: struct layouts, the rotation's frequencies, the
masks of trees, every refusal, and the oracle's 8-bit rounding (CPU only)."""
from __future__ import annotations

import ctypes
import math
import os
import random

import pytest
import torch

from oracle import cacheops as oracle
from paper_2608_28099_amd import binding, ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sp_probe.h")
BAD, UNSUPPORTED, CAPACITY = -1, -2, -6

pytestmark = pytest.mark.skipif(not os.path.exists(binding.LIB_PATH),
                                reason="libsp_probe.so not built (run __graft_entry__.build())")


def test_struct_layouts_match_the_c_compiler(tmp_path):
    import shutil
    import subprocess
    if shutil.which("gcc") is None:
        pytest.skip("gcc not available")
    names = ("sp_kv_store", "sp_rows", "sp_rotary_config", "sp_rotary", "sp_tree_config", "sp_tree")
    lines = ['#include <stdio.h>', '#include <stddef.h>', f'#include "{HEADER}"', "int main(void) {"]
    for n in names:
        lines.append(f'  printf("{n} %zu\\n", sizeof({n}));')
        lines += [f'  printf("{n}.{f[0]} %zu\\n", offsetof({n}, {f[0]}));' for f in getattr(binding, n)._fields_]
    lines.append("  return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run(["gcc", "-std=c99", "-o", str(exe), str(src)], check=True)
    out = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for n in names:
        cls = getattr(binding, n)
        assert int(out[n]) == ctypes.sizeof(cls), n
        for f in cls._fields_:
            assert int(out[f"{n}.{f[0]}"]) == getattr(cls, f[0]).offset, (n, f[0])


@pytest.mark.parametrize("dim,kw", [
    (128, {}), (64, {"base": 1e6}), (2, {}), (128, {"scaling": "linear", "factor": 3.0}),
    (90, {"scaling": "ntk", "factor": 4.0}), (128, {"scaling": "yarn", "factor": 4.0, "original": 32768.0}),
    (64, {"scaling": "yarn", "factor": 16.0, "original": 4096.0, "base": 1e6}), (32, {"base": 0.5})])
def test_frequencies_follow_the_definition(dim, kw):
    theta, scale = oracle.frequencies(dim, **kw)
    kw = dict(kw)
    kw["original_positions"] = kw.pop("original", 0)
    rot = ops.make_rotary(128, rotary_dim=dim, **kw)
    got = torch.tensor(list(rot.turns)[:dim // 2], dtype=torch.float64) * 2 * math.pi
    # a few roundings of 2^-53 each in pow, its argument, the division and the product
    assert torch.allclose(got, theta, rtol=2e-15, atol=0)
    assert rot.scale == pytest.approx(scale, rel=2 ** -23)
    assert all(t == 0 for t in list(rot.turns)[dim // 2:])


def test_custom_frequencies():
    rot = ops.make_rotary(64, rotary_dim=6, scaling="custom", frequencies=[1.0, 0.0, -0.25], attn_factor=1.5)
    assert list(rot.turns)[:3] == [1.0 / (2 * math.pi), 0.0, -0.25 / (2 * math.pi)] and rot.scale == 1.5


def test_rotations_that_are_refused():
    lib = binding.load()
    good = dict(head_dim=128, rotary_dim=128, layout=0, scaling=0, base=10000.0, factor=2.0, original_positions=4096.0)
    out = binding.sp_rotary()

    def init(**kw):
        return lib.sp_probe_rotary_init(ctypes.byref(binding.sp_rotary_config(**dict(good, **kw))), ctypes.byref(out))

    assert init() == 0
    assert init(head_dim=96) == UNSUPPORTED
    for kw in (dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=130), dict(layout=2), dict(scaling=5),
               dict(scaling=-1), dict(base=0.0), dict(base=math.inf), dict(base=math.nan), dict(base=1e-30),
               dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan), dict(scaling=2, rotary_dim=2),
               dict(scaling=3, original_positions=0.0), dict(scaling=3, beta_fast=1.0, beta_slow=2.0),
               dict(scaling=3, attn_factor=-1.0), dict(scaling=4),):
        assert init(**kw) == BAD, kw
    assert lib.sp_probe_rotary_init(None, ctypes.byref(out)) == BAD
    assert lib.sp_probe_rotary_init(ctypes.byref(binding.sp_rotary_config(**good)), None) == BAD
    with pytest.raises(ValueError):
        ops.make_rotary(128, layout="other")
    with pytest.raises(ValueError):
        ops.make_rotary(128, scaling="custom", frequencies=[1.0])
    with pytest.raises(binding.ProbeError):
        ops.make_rotary(128, scaling="custom", frequencies=[math.nan] * 64)


P = 0x10000  # a pointer that no refused call reads


def rows(heads, data=P, **kw):
    return binding.sp_rows(data=data, stride_row=heads * 128, stride_head=128, n_heads=heads, **kw)


def store(dtype=binding.SP_BF16, **kw):
    kv = dict(k_base=P, v_base=P, num_blocks=8, k_stride_block=4096, k_stride_head=2048, v_stride_block=4096,
              v_stride_head=2048, block_size=16, max_blocks_per_seq=4, batch=2)
    top = dict(dtype=dtype, n_kv_heads=2, head_dim=128)
    if dtype == binding.SP_E4M3:
        top.update(k_exponents=P, v_exponents=P, exponent_stride_block=32, exponent_stride_head=16)
    for k, v in kw.items():
        (kv if k in kv else top)[k] = v
    return binding.sp_kv_store(kv=binding.sp_kv_cache(**kv), **top)


BAD_STORES = [dict(dtype=3), dict(n_kv_heads=0), dict(k_base=None), dict(v_base=P + 8), dict(num_blocks=0),
              dict(k_stride_block=4095), dict(v_stride_head=1024), dict(block_size=24), dict(block_size=8),
              dict(max_blocks_per_seq=0), dict(batch=-1), dict(reserved=1)]


def test_stores_that_are_refused():
    lib = binding.load()
    kr = rows(2)

    def write(s, table=P):
        return lib.sp_probe_cache_write(ctypes.byref(s), table, 1, 4, P, P, None, 4, ctypes.byref(kr),
                                        ctypes.byref(kr), None, None)

    def read(s, table=P):
        return lib.sp_probe_cache_read(ctypes.byref(s), table, 1, 4, P, P, ctypes.byref(kr), ctypes.byref(kr), None)

    for f in (write, read):
        for kw in BAD_STORES:
            assert f(store(**kw)) == BAD, kw
        assert f(store(head_dim=96)) == UNSUPPORTED
        assert f(store(batch=3), None) == BAD      # contiguous storage needs batch * blocks blocks
        for kw in (dict(k_exponents=None), dict(v_exponents=P + 1), dict(exponent_stride_block=8),
                   dict(exponent_stride_head=0), dict(k_stride_head=2056)):
            assert f(store(binding.SP_E4M3, **kw)) == BAD, kw
    assert lib.sp_probe_cache_write(None, P, 1, 4, P, P, None, 4, ctypes.byref(kr), ctypes.byref(kr), None, None) == BAD


def test_row_arguments_that_are_refused():
    lib = binding.load()
    s = ctypes.byref(store())
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    rot64 = ops.make_rotary(64)

    def write(dtype=1, n=4, seq=P, pos=P, src=None, n_src=4, k=rows(2), v=rows(2), rot=None):
        return lib.sp_probe_cache_write(s, P, dtype, n, seq, pos, src, n_src, r(k), r(v), r(rot), None)

    def read(dtype=1, n=4, seq=P, pos=P, k=rows(2), v=rows(2)):
        return lib.sp_probe_cache_read(s, P, dtype, n, seq, pos, r(k), r(v), None)

    for f in (write, read):
        for kw in (dict(dtype=2), dict(n=-1), dict(seq=None), dict(pos=None), dict(pos=P + 2), dict(k=rows(3)),
                   dict(v=rows(2, None)), dict(k=rows(2, P + 1)), dict(v=rows(2, reserved=1))):
            assert f(**kw) == BAD, kw
        assert f(n=0, seq=None, pos=None, k=None, v=None) == 0
    assert write(k=None) == BAD and write(v=None) == BAD and write(src=P + 1) == BAD and write(n_src=-1) == BAD
    assert write(rot=rot64) == BAD                 # of another head width
    assert write(n_src=0) == 0 and read(k=None, v=None) == 0

    rot = ops.make_rotary(128)
    bad = binding.sp_rotary(head_dim=128, rotary_dim=5)

    def rotary(rot=rot, dtype=1, n=4, pos=P, q=rows(8), qo=rows(8), k=rows(2), ko=rows(2)):
        return lib.sp_probe_rotary(r(rot), dtype, 0, n, pos, r(q), r(qo), r(k), r(ko), None)

    for kw in (dict(rot=None), dict(rot=bad), dict(dtype=2), dict(n=-1), dict(pos=None), dict(q=None), dict(qo=None),
               dict(ko=None), dict(k=None), dict(qo=rows(4)), dict(q=rows(0), qo=rows(0)), dict(q=rows(8, P + 1)),
               dict(ko=rows(2, None))):
        assert rotary(**kw) == BAD, kw
    assert rotary(q=rows(5000), qo=rows(5000)) == UNSUPPORTED
    assert rotary(n=0, pos=None) == 0


def test_trees_that_are_refused():
    lib = binding.load()
    cfg0 = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=1, kv_dtype=1, max_nodes=8, max_batch=2, max_seq_len=64)

    def need(**kw):
        return lib.sp_probe_tree_workspace_bytes(ctypes.byref(binding.sp_tree_config(**dict(cfg0, **kw))))

    def call(st=None, lens=P, ws=P, ws_bytes=1 << 40, table=P, tree=True, cfg=None, **kw):
        t = binding.sp_tree(n_nodes=4, q=rows(8), k=rows(2), v=rows(2), out=rows(8))
        for k, v in kw.items():
            setattr(t, k, v)
        c = binding.sp_tree_config(**dict(cfg0, **(cfg or {})))
        return lib.sp_probe_tree_attention(ctypes.byref(c), ctypes.byref(st or store()), lens, table,
                                           ctypes.byref(t) if tree else None, ws, ws_bytes, None)

    assert need() > 0
    for kw in (dict(n_q_heads=0), dict(n_q_heads=9), dict(dtype=2), dict(kv_dtype=3), dict(max_nodes=0),
               dict(max_batch=0), dict(max_seq_len=-1), dict(scale=-1.0), dict(scale=math.inf), dict(reserved=1)):
        assert need(**kw) == 0 and call(cfg=kw) == BAD, kw
    for kw in (dict(head_dim=96), dict(dtype=0), dict(kv_dtype=0), dict(max_nodes=257), dict(max_batch=70000)):
        assert need(**kw) == 0 and call(cfg=kw) == UNSUPPORTED, kw
    for kw in BAD_STORES:
        assert call(store(**kw)) == BAD, kw
    assert call(store(binding.SP_E4M3)) == BAD     # not the config's storage
    assert call(tree=False) == BAD and call(lens=None) == BAD and call(lens=P + 2) == BAD
    assert call(ws=None) == BAD and call(ws=P + 8) == BAD and call(ws_bytes=need() - 1) == BAD
    assert call(n_nodes=0) == BAD and call(n_nodes=9) == CAPACITY and call(cfg=dict(max_batch=1)) == CAPACITY
    assert call(cfg=dict(max_seq_len=65)) == BAD   # a block table's row holds 64 tokens
    assert call(mask=P, mask_words=0) == BAD and call(mask=P + 1, mask_words=1) == BAD
    assert call(mask=P, mask_words=1, mask_stride=-1) == BAD
    for name, heads in (("q", 8), ("k", 2), ("v", 2), ("out", 8)):
        assert call(**{name: rows(heads + 1)}) == BAD and call(**{name: rows(heads, None)}) == BAD
        assert call(**{name: rows(heads, P + 1)}) == BAD
    assert call(counts=P + 1) == BAD and call(lse=P + 2) == BAD
    assert call(store(batch=0), lens=None) == 0


def test_wrong_tensors_raise_before_the_library():
    k = torch.zeros(4, 2, 2048, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ops.PagedCache(k, k.float(), 16, batch=1)
    with pytest.raises(ValueError):
        ops.PagedCache(k, k, 16)
    with pytest.raises(ValueError):
        ops.PagedCache(k.to(torch.float8_e4m3fn), k.to(torch.float8_e4m3fn), 16, batch=1)
    with pytest.raises(ValueError):
        ops.PagedCache(k, k, 16, torch.zeros(1, 2, dtype=torch.int64))
    cache = ops.PagedCache(k, k, 16, torch.zeros(1, 2, dtype=torch.int32))
    x = torch.zeros(1, 3, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):                # not on the GPU
        ops.tree_attention(cache, torch.zeros(1, dtype=torch.int32), x, x, x)
    with pytest.raises(ValueError):
        ops.rotary(ops.make_rotary(128), torch.zeros(3, dtype=torch.int32), x[0])


def test_tree_masks():
    rng = random.Random(3)
    for t in (1, 2, 31, 32, 33, 100):
        parents = [[rng.randint(-1, i - 1) for i in range(t)] for _ in range(3)]
        words = ops.tree_mask(parents)
        assert words.shape == (3, t, -(-t // 32)) and words.dtype == torch.int32
        for b in range(3):
            for i in range(t):
                want, at = set(), i
                while at >= 0:
                    want.add(at)
                    at = parents[b][at]
                got = {j for j in range(32 * words.shape[2]) if (int(words[b, i, j // 32]) >> (j % 32)) & 1}
                assert got == want
    with pytest.raises(ValueError):
        ops.tree_mask([0])


def test_the_oracle_rounds_as_e4m3():
    torch.manual_seed(1)
    x = torch.randn(64, 32, dtype=torch.float64) * torch.exp2(torch.randint(-20, 20, (64, 1)).double())
    x[0] = 0
    x[1] *= 1e-40
    v, byte = oracle.quantise(x.float())
    e = byte.double() - 127
    ref = (x.float().double() / torch.exp2(e)[:, None]).float().to(torch.float8_e4m3fn).double()
    assert torch.equal(v, ref)
    assert float(v.abs().max()) <= 448 and bool((v[2:].abs().amax(-1) > 223).all())
    w, _ = oracle.quantise(torch.tensor([[math.inf, -1.0, math.nan, 2.0]]))
    assert torch.isnan(w[0, [0, 2]]).all() and w[0, [1, 3]].tolist() == [-128.0, 256.0]


def test_the_longest_context():
    lib = binding.load()
    cfg = binding.sp_tree_config(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=1, kv_dtype=1, max_nodes=8, max_batch=1,
                                 max_seq_len=1 << 30)
    assert lib.sp_probe_tree_workspace_bytes(ctypes.byref(cfg)) > 0
    cfg.max_seq_len += 1
    assert lib.sp_probe_tree_workspace_bytes(ctypes.byref(cfg)) == 0
    t = binding.sp_tree(n_nodes=4, q=rows(8), k=rows(2), v=rows(2), out=rows(8))
    assert lib.sp_probe_tree_attention(ctypes.byref(cfg), ctypes.byref(store()), P, P, ctypes.byref(t), P, 1 << 40, None) == UNSUPPORTED
    # a table whose rows reach further gives attention that many tokens at most
    table = torch.zeros((1, 1 << 16), dtype=torch.int32)
    assert ops.PagedCache.allocate(torch.bfloat16, 1, 1, 64, 1 << 15, table, device="cpu").capacity == 1 << 30


def test_rows_of_single_nodes():
    """[batch, 1, heads, hd] taken from packed projections: the rows' step is the batch's stride."""
    packed = torch.zeros(3, 12, 64)
    r = ops._rows(packed[:, :8].unsqueeze(1), "q", 64, torch.float32, packed.device)
    assert (r.stride_row, r.stride_head, r.n_heads) == (12 * 64, 64, 8)
    r = ops._rows(packed.view(3, 1, 12, 64)[:, :, 8:], "k", 64, torch.float32, packed.device)
    assert (r.stride_row, r.n_heads) == (12 * 64, 4)
    r = ops._rows(packed[None, :, :8], "q", 64, torch.float32, packed.device)  # one sequence of three nodes
    assert (r.stride_row, r.n_heads) == (12 * 64, 8)
    with pytest.raises(ValueError):
        ops._rows(torch.zeros(2, 4, 12, 64)[:, :3], "q", 64, torch.float32, packed.device)


def test_rows_without_a_source():
    lib = binding.load()
    nothing = rows(2, None)
    for n_src, want in ((0, 0), (1, BAD)):
        assert lib.sp_probe_cache_write(ctypes.byref(store()), P, binding.SP_BF16, 3, P, P, P, n_src, ctypes.byref(nothing),
                                        ctypes.byref(nothing), None, None) == want


def test_the_most_rows():
    lib = binding.load()
    rot = ops.make_rotary(128)
    q, k = rows(2), rows(2)
    n = 1 << 26
    assert lib.sp_probe_rotary(rot, binding.SP_BF16, 0, n, P, q, q, None, None, None) == UNSUPPORTED
    assert lib.sp_probe_cache_write(store(), P, binding.SP_BF16, n, P, P, None, n, k, k, None, None) == UNSUPPORTED
    assert lib.sp_probe_cache_read(store(), P, binding.SP_BF16, n, P, P, k, k, None) == UNSUPPORTED
