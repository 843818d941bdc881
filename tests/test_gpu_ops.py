"""The cache operators (rotary positions, cache writing and reading, tree attention)
against their fp64 definitions, at the sizes, layouts and masks where they could go wrong."""
from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from oracle import cacheops as oracle
from paper_2608_28099_amd import binding, ops

pytestmark = pytest.mark.gpu

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # of a rounding, relative


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()
    return torch.device("cuda:0")


def randn(gen, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=gen) * std).to(dtype)


def seeded(seed):
    return torch.Generator().manual_seed(seed)


# ---------------------------------------------------------------- rotary

ROTATIONS = [
    (128, dict(), 128, "half"), (128, dict(), 128, "interleaved"), (64, dict(scaling="linear", factor=2.0), 32, "half"),
    (64, dict(base=1e6), 64, "interleaved"), (128, dict(scaling="yarn", factor=4.0, original=4096.0), 64, "half"),
    (128, dict(scaling="ntk", factor=8.0), 88, "interleaved"), (128, dict(), 90, "half"), (64, dict(), 2, "half"),
    (128, dict(base=0.5), 32, "half"), (128, dict(), 126, "interleaved")]


def make_rot(hd, kw, dim, layout):
    kw = dict(kw)
    return ops.make_rotary(hd, rotary_dim=dim, layout=layout, original_positions=kw.pop("original", 0), **kw)


def rotation_error(y, x, ref, theta, scale, layout, positions):
    """|y - ref| over what the arithmetic allows: the cosines and sines, their scale, two products and a sum
    in fp32 (half a step each, so 5 * 2^-24 of |a| + |b|), angles a few 2^-53 of themselves off, one rounding of the result."""
    half = len(theta)
    mag = torch.zeros_like(ref)
    for p in range(half):
        i, j = (p, p + half) if layout == "half" else (2 * p, 2 * p + 1)
        mag[..., i] = mag[..., j] = scale * (x[..., i].abs() + x[..., j].abs()).double()
    ang = positions.double().abs().max() * theta.abs().max() * 2.0 ** -51
    tol = HALF_STEP[y.dtype] * ref.abs() + (5 * 2.0 ** -24 + ang) * (1 + HALF_STEP[y.dtype]) * mag
    return float(((y.double() - ref).abs() / (tol + 1e-300)).max())


@pytest.mark.parametrize("hd,kw,dim,layout", ROTATIONS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,far", [(1, 1), (7, 300), (130, 1000003)])
def test_rotary(dev, hd, kw, dim, layout, dtype, rows, far):
    if kw.get("base") == 0.5 and far > 1000:
        far = 1000
    gen = seeded(rows + dim)
    x = randn(gen, rows, 7, hd, dtype=dtype)
    pos = torch.randint(0, far, (rows,), generator=gen, dtype=torch.int32)
    pos[-1] = far - 1
    theta, scale = oracle.frequencies(dim, **kw)
    rot = make_rot(hd, kw, dim, layout)
    xd, pd = x.to(dev), pos.to(dev)
    q, k = xd[:, :4], xd[:, 4:6]
    for transpose in (False, True):
        ref = oracle.rotate(x, pos, theta, scale, layout, transpose)
        yq, yk = ops.rotary(rot, pd, q, k, transpose=transpose)
        y = torch.cat([yq, yk], 1).cpu()
        assert rotation_error(y, x[:, :6], ref[:, :6], theta, scale, layout, pos) <= 1
        assert torch.equal(y[..., dim:], x[:, :6, dim:])
        z = xd.clone()                                   # in place, one array
        assert ops.rotary(rot, pd, z[:, :4], out=z[:, :4], transpose=transpose).data_ptr() == z.data_ptr()
        assert torch.equal(z[:, :4], yq) and torch.equal(z[:, 4:], xd[:, 4:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rotary_of_odd_strides_and_padding(dev, dtype):
    """Heads that are not 16-byte aligned, rows in another order in memory, rows at negative positions."""
    gen = seeded(5)
    rot = ops.make_rotary(64, rotary_dim=24, layout="half")
    theta, scale = oracle.frequencies(24)
    base = randn(gen, 9 * 3 * 67 + 1, dtype=dtype)
    x = base[1:].view(9, 3, 67)[..., :64]
    pos = torch.tensor([3, -1, 0, 77, -5, 2, 1, 100, 6], dtype=torch.int32)
    big = base.to(dev)
    xd = big[1:].view(9, 3, 67)[..., :64]
    out = torch.full((3, 9, 64), 7.0, dtype=dtype, device=dev).transpose(0, 1)
    ops.rotary(rot, pos.to(dev), xd, out=out)
    got, ref = out.cpu(), oracle.rotate(x, pos, theta, scale)
    live = pos >= 0
    assert rotation_error(got[live], x[live], ref[live], theta, scale, "half", pos[live]) <= 1
    assert torch.all(got[~live] == 7.0) and torch.equal(big.cpu(), base)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotary_gradient(dev, layout):
    """The transposed rotation is the gradient: against differences of the rotation, which is linear
    (so a difference over a step of 1 is exact up to the rounding of both sides)."""
    gen = seeded(9)
    rot = ops.make_rotary(64, rotary_dim=16, layout=layout, scaling="yarn", factor=4.0, original_positions=64)
    pos = torch.tensor([0, 5, 1000], dtype=torch.int32, device=dev)
    x, gy = randn(gen, 3, 2, 64).to(dev), randn(gen, 3, 2, 64).to(dev)
    gx = ops.rotary(rot, pos, gy, transpose=True)
    y = ops.rotary(rot, pos, x)
    for d in range(0, 64, 5):
        step = x.clone()
        step[..., d] += 1.0
        diff = ((ops.rotary(rot, pos, step) - y).double() * gy.double()).sum(-1)
        # y and its step: values up to 8, each rounded (and so are the sums that make x + 1): 2^-20 over 2 terms of |gy| <= 4
        assert torch.all((diff - gx[..., d].double()).abs() <= 16 * 2.0 ** -20), d


# ---------------------------------------------------------------- the cache

def make_cache(dev, dtype, lens, nkv, hd, block, seed=0, extra=3, fill=None, contiguous=False):
    per = [-(-n // block) for n in lens]
    most = max(max(per), 1)
    if contiguous:
        table, blocks = None, most * len(lens)
    else:
        blocks = sum(per) + extra
        order = torch.randperm(blocks, generator=seeded(seed)).int()
        table = torch.full((len(lens), most), int(order[-1]), dtype=torch.int32)
        at = 0
        for b, n in enumerate(per):
            table[b, :n] = order[at:at + n]
            at += n
        table = table.to(dev)
    cache = ops.PagedCache.allocate(dtype, blocks, nkv, hd, block, table, len(lens) if contiguous else None, dev)
    if fill is not None:
        cache.k.copy_(torch.full(cache.k.shape, fill, device=dev).to(dtype))
        cache.v.copy_(torch.full(cache.v.shape, fill, device=dev).to(dtype))
        if cache.k_exponents is not None:
            cache.k_exponents.fill_(255)
            cache.v_exponents.fill_(255)
    return cache


def contents(cache, which):
    """[blocks, heads, block, hd] on the CPU as stored (8-bit values without their exponents)."""
    t = (cache.k if which == "k" else cache.v).cpu()
    raw = t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t
    bs, hd = cache.block_size, cache.head_dim
    if which == "v":
        return raw.reshape(*raw.shape[:2], hd, bs).transpose(2, 3).contiguous().view(t.dtype)
    x = 16 // t.element_size()
    return raw.reshape(*raw.shape[:2], hd // x, bs, x).permute(0, 1, 3, 2, 4).reshape(*raw.shape[:2], bs, hd).contiguous().view(t.dtype)


def slots(cache, seq, pos):
    table = (cache.block_table.cpu() if cache.block_table is not None
             else torch.arange(cache.batch * cache.max_blocks).reshape(cache.batch, -1))
    return table[seq.long(), pos.long() // cache.block_size].long(), pos.long() % cache.block_size


def tokens(lens, starts=None):
    seq = torch.cat([torch.full((n,), b, dtype=torch.int32) for b, n in enumerate(lens)])
    pos = torch.cat([torch.arange(n, dtype=torch.int32) + (0 if starts is None else starts[b]) for b, n in enumerate(lens)])
    return seq, pos


STORES = [torch.float32, torch.bfloat16, torch.float8_e4m3fn]


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("hd,block,lens,starts,shuffle", [
    (128, 16, (1,), (0,), False), (64, 16, (70, 0, 3, 64), (0, 0, 5, 16), False), (128, 32, (130, 17), (3, 31), False),
    (128, 16, (45, 20), (7, 0), True), (64, 256, (100, 33), (60, 250), False)])
def test_cache_write_and_read(dev, store, dtype, hd, block, lens, starts, shuffle):
    gen, nkv = seeded(hd + block), 3
    seq, pos = tokens(lens, starts)
    n = len(seq)
    if shuffle:
        order = torch.randperm(n, generator=gen)
        seq, pos = seq[order], pos[order]
    cache = make_cache(dev, store, [a + b for a, b in zip(lens, starts)], nkv, hd, block, contiguous=block == 256)
    x = randn(gen, n, 8, hd, dtype=dtype) * torch.exp2(torch.randint(-9, 9, (n, 8, 1), generator=gen)).to(dtype)
    k, v = x[:, 1:4], x[:, 5:8]
    xd = x.to(dev)
    sd, pd = seq.to(dev), pos.to(dev)
    ops.cache_write(cache, sd, pd, xd[:, 1:4], xd[:, 5:8])
    blk, slot = slots(cache, seq, pos)
    used = torch.zeros(cache.num_blocks, block, dtype=torch.bool)
    used[blk, slot] = True
    for which, want in (("k", k), ("v", v)):
        got = contents(cache, which)
        if store == torch.float8_e4m3fn:
            val, byte = oracle.quantise(want)
            exps = (cache.k_exponents if which == "k" else cache.v_exponents).cpu()
            assert torch.equal(exps[blk, :, slot].long(), byte)
            assert torch.equal(got.float()[blk, :, slot].double(), val)
            assert torch.all(exps.transpose(1, 2)[~used] == 127)
        else:
            assert torch.equal(got[blk, :, slot], want.to(store))
        assert torch.all(got.float().transpose(1, 2)[~used] == 0)
    for out in (torch.float32, torch.bfloat16):
        kr, vr = ops.cache_read(cache, sd, pd, out)
        for got, want in ((kr, k), (vr, v)):
            if store == torch.float8_e4m3fn:
                val, byte = oracle.quantise(want)
                want = val * torch.exp2(byte.double() - 127)[..., None]
            else:
                want = want.to(store)
            assert torch.equal(got.cpu(), want.to(out))
    only = torch.zeros((n, nkv, hd), dtype=torch.float32, device=dev)   # one of the two; a token twice
    twice = torch.zeros_like(only)
    ops.cache_read(cache, sd, pd, k=only)
    ops.cache_read(cache, sd[:1].expand(n).contiguous(), pd[:1].expand(n).contiguous(), v=twice)
    assert torch.equal(only, ops.cache_read(cache, sd, pd, torch.float32)[0])
    assert torch.equal(twice, ops.cache_read(cache, sd[:1], pd[:1], torch.float32)[1].expand(n, -1, -1))


@pytest.mark.parametrize("store", STORES)
def test_rows_out_of_range_are_skipped(dev, store):
    gen = seeded(4)
    lens = (40, 40)
    cache = make_cache(dev, store, lens, 2, 64, 16)
    cache.block_table[1, 1] = cache.num_blocks            # a page that is not in the pool
    cache.block_table[1, 2] = -1
    seq = torch.tensor([0, 0, 2, -1, 0, 1, 1, 1, 0, 0], dtype=torch.int32)
    pos = torch.tensor([0, -1, 1, 1, 48, 3, 17, 33, 5, 6], dtype=torch.int32)
    src = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, 99, -1], dtype=torch.int32)
    live = torch.tensor([1, 0, 0, 0, 0, 1, 0, 0, 0, 0], dtype=torch.bool)
    x = randn(gen, 10, 2, 64)
    args = cache, seq.to(dev), pos.to(dev)
    ops.cache_write(*args, x.to(dev), x.to(dev), src_rows=src.to(dev))
    for which in "kv":
        assert int((contents(cache, which).float() != 0).any(-1).any(1).sum()) == 2
    k = torch.full((10, 2, 64), 9.0, device=dev)
    v = k.clone()
    ops.cache_read(*args, k=k, v=v)
    ok = live.clone()
    ok[8:] = True                                          # slots that exist, never written
    for t in (k.cpu(), v.cpu()):
        assert torch.all(t[~ok] == 9.0) and torch.all(t[8:] == 0)
        if store == torch.float32:
            assert torch.equal(t[live], x[live])


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("layout,dim,hd", [("half", 128, 128), ("interleaved", 64, 64), ("half", 34, 128), ("interleaved", 6, 128)])
def test_keys_rotated_as_they_are_written(dev, store, layout, dim, hd):
    gen = seeded(dim)
    starts, lens = (100, 70000), (50, 3)
    cache = make_cache(dev, store, [a + b for a, b in zip(lens, starts)], 2, hd, 16)
    seq, pos = tokens(lens, starts)
    n = len(seq)
    x = randn(gen, n, 4, hd)
    src = torch.randperm(n, generator=gen).int()
    theta, scale = oracle.frequencies(dim)
    xd = x.to(dev)
    ops.cache_write(cache, seq.to(dev), pos.to(dev), xd[:, :2], xd[:, 2:], src_rows=src.to(dev),
                    rotary=ops.make_rotary(hd, rotary_dim=dim, layout=layout))
    k, v = ops.cache_read(cache, seq.to(dev), pos.to(dev), torch.float32)
    xk = x[src.long(), :2]
    ref = oracle.rotate(xk, pos, theta, scale, layout)
    if store == torch.float8_e4m3fn:
        # one rounding of e4m3 (2^-4 of the value, or half the smallest step, 2^-10 of the scale) of
        # a value 6 * 2^-24 off
        scale8 = torch.exp2(oracle.quantise(ref)[1].double() - 127)[..., None]
        err = (k.cpu().double() - ref).abs()
        assert torch.all(err <= ref.abs() * 2.0 ** -4 * (1 + 1e-5) + scale8 * 2.0 ** -10 + 1e-5 * 2.0 ** -3)
        assert torch.equal(v.cpu().double(), (lambda w, b: w * torch.exp2(b.double() - 127)[..., None])(*oracle.quantise(x[src.long(), 2:])))
    else:
        got = k.cpu()
        assert rotation_error(got.to(store), xk, ref, theta, scale, layout, pos) <= 1
        assert torch.equal(v.cpu(), x[src.long(), 2:].to(store).float())


def test_8_bit_rows_of_odd_values(dev):
    """Zeros, the smallest and largest magnitudes, ties, NaN and infinities."""
    x = torch.zeros(9, 1, 64)
    x[1, 0, :4] = torch.tensor([1e-45, -1e-40, 2.0 ** -126, 0.0])
    x[2, 0, :4] = torch.tensor([3.3e38, -3.3e38, 1e30, 1.0])
    x[3, 0, :4] = torch.tensor([math.inf, -1.0, math.nan, 2.0])
    x[4, 0, :] = math.nan
    x[5, 0, :8] = torch.tensor([448.0, 17.0, 18.0, 19.0, 21.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10])
    x[6, 0, :8] = torch.tensor([448.0, -17.0, 25.0, 27.0, 232.0, 5 * 2.0 ** -10, -(2.0 ** -10), 7 * 2.0 ** -10])
    x[7, 0, :3] = torch.tensor([448.0001, 224.0, 1.0])
    x[8, 0, :3] = torch.tensor([-0.0, 1.75, -1.75])
    cache = make_cache(dev, torch.float8_e4m3fn, (9,), 1, 64, 16)
    seq, pos = tokens((9,))
    ops.cache_write(cache, seq.to(dev), pos.to(dev), x.to(dev), x.to(dev))
    val, byte = oracle.quantise(x)
    for which, e in (("k", cache.k_exponents), ("v", cache.v_exponents)):
        got = contents(cache, which).float()[0 if cache.num_blocks == 1 else int(cache.block_table[0, 0]), :, :9].transpose(0, 1).double()
        assert torch.equal(torch.isnan(got), torch.isnan(val))
        # what a denormal fp32 magnitude rounds to is below half of the smallest step: 0
        assert torch.equal(got.nan_to_num(), val.nan_to_num())
        assert torch.equal(e.cpu()[int(cache.block_table[0, 0]), 0, :9].long(), byte[:, 0])


# ---------------------------------------------------------------- tree attention

def random_tree(gen, t):
    parents = [-1] + [int(torch.randint(max(-1, i - 5), i, (1,), generator=gen)) for i in range(1, t)]
    see = torch.zeros(t, t, dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            see[i] = see[p]
        see[i, i] = True
    return parents, see


def words_of(see):
    t = see.shape[-1]
    w = -(-t // 32)
    full = torch.zeros(*see.shape[:-1], 32 * w, dtype=torch.int64)
    full[..., :t] = see
    words = (full.view(*see.shape[:-1], w, 32) << torch.arange(32)).sum(-1)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32)


def dense(cache, b, n):
    """The cache's keys and values of sequence b, [nkv, n, hd] in fp64 as they stand."""
    seq, pos = torch.full((n,), b, dtype=torch.int32), torch.arange(n, dtype=torch.int32)
    blk, slot = slots(cache, seq, pos)
    out = []
    for which, e in (("k", cache.k_exponents), ("v", cache.v_exponents)):
        c = contents(cache, which).float()[blk, :, slot].double()
        if e is not None:
            c = c * torch.exp2(e.cpu()[blk, :, slot].double() - 127)[..., None]
        out.append(c.transpose(0, 1))
    return out


class Tree:
    """Inputs of a call, every token of the cache written by the operator, slots past the ends NaN."""

    def __init__(self, dev, store, lens, t, nq, nkv, hd, block, seed=0, std=1.0, contiguous=False):
        gen = seeded(seed)
        self.dtype = torch.float32 if store == torch.float32 else torch.bfloat16
        self.lens, self.t, self.nq, self.nkv, self.hd, self.dev = lens, t, nq, nkv, hd, dev
        self.cache = make_cache(dev, store, lens, nkv, hd, block, seed, fill=math.nan, contiguous=contiguous)
        seq, pos = tokens(lens)
        x = randn(gen, len(seq), 2 * nkv, hd, dtype=self.dtype)
        xd = x.to(dev)
        if len(seq):
            ops.cache_write(self.cache, seq.to(dev), pos.to(dev), xd[:, :nkv], xd[:, nkv:])
        self.x = randn(gen, len(lens), t, nq + 2 * nkv, hd, dtype=self.dtype)
        self.x[:, :, :nq] *= std
        trees = [random_tree(gen, t) for _ in lens]
        self.see = torch.stack([s for _, s in trees])
        self.parents = [p for p, _ in trees]
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device=dev)

    def qkv(self, x=None):
        x = (self.x if x is None else x).to(self.dev)
        return x[:, :, :self.nq], x[:, :, self.nq:self.nq + self.nkv], x[:, :, self.nq + self.nkv:]

    def check(self, out, lse=None, see=None, counts=None, scale=None, x=None, sequences=None):
        """Against the definition.  Roundings: each weight (bf16: 2^-8 of itself; fp32: none) and the result; a score of
        hd products is off by at most hd 2^-24 of sum |q||k| and moves its weight by as much (and the sum's,
        so twice), an exponential by 2^-22, sums of n terms by n 2^-24 each of sum w|v|."""
        x = self.x if x is None else x
        see = self.see if see is None else see
        out = out.cpu()
        for b, n in enumerate(self.lens):
            if sequences is not None and b not in sequences:
                continue
            c = self.t if counts is None else counts[b]
            if c == 0:
                continue
            kc, vc = dense(self.cache, b, n)
            q, k, v = x[b, :c, :self.nq], x[b, :c, self.nq:self.nq + self.nkv], x[b, :c, self.nq + self.nkv:]
            ref, rl, mag, big = oracle.tree_attention(q, kc, vc, k, v, see[b, :c, :c], scale)
            eps = 2 * (self.hd * 2.0 ** -24 * big + 2.0 ** -22) + 2 * (n + c + 8) * 2.0 ** -24
            u = 0.0 if self.dtype == torch.float32 else 2.0 ** -8
            tol = mag * (u + eps) * (1 + 2.0 ** -6) + HALF_STEP[self.dtype] * ref.abs() + 1e-30
            err = (out[b, :c].double() - ref).abs() / tol
            assert torch.isfinite(out[b, :c].float()).all() and float(err.max()) <= 1, (b, float(err.max()))
            if lse is not None:
                got = lse[b, :c].cpu().double()
                empty = rl == -math.inf
                assert torch.equal(got == -math.inf, empty)
                off = (got - rl)[~empty].abs()
                assert torch.all(off <= eps + 2.0 ** -22 * (1 + rl[~empty].abs())), float(off.max())


CASES = [  # lens, nodes, query heads, KV heads, hd, block
    ((256, 256), 4, 4, 2, 64, 16),
    ((0, 1, 15, 16, 17, 31, 32, 33), 3, 8, 2, 128, 16),
    ((63, 64, 65, 517, 100), 13, 8, 2, 128, 16),
    ((47, 300, 1000), 8, 10, 2, 128, 32),
    ((2048,), 60, 8, 2, 128, 64),
    ((130, 5), 1, 8, 8, 64, 16),
    ((77,), 100, 4, 1, 64, 16),
    ((40, 0), 200, 6, 3, 128, 16),
    ((5000, 3), 2, 2, 2, 128, 16),
    ((1300, 700), 33, 12, 1, 128, 512),
]


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lens,t,nq,nkv,hd,block", CASES)
def test_tree_attention(dev, store, lens, t, nq, nkv, hd, block):
    c = Tree(dev, store, lens, t, nq, nkv, hd, block, seed=t)
    q, k, v = c.qkv()
    lse = torch.zeros((len(lens), t, nq), device=dev)
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(c.see).to(dev), max_seq_len=max(lens), lse=lse)
    c.check(out, lse)
    again = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=ops.tree_mask(c.parents).to(dev), max_seq_len=max(lens))
    assert torch.equal(out, again)                       # the same bits from run to run


@pytest.mark.parametrize("store", STORES)
def test_peaked_scores(dev, store):
    """Scores of a few hundred: the maximum moves and everything else vanishes."""
    c = Tree(dev, store, (333, 40), 9, 4, 2, 128, 16, seed=3, std=25.0)
    q, k, v = c.qkv()
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(c.see).to(dev), max_seq_len=333)
    c.check(out)


@pytest.mark.parametrize("store", STORES)
def test_chain_scale_and_default_length(dev, store):
    """No mask: each node sees those up to itself.  A scale of the caller's, the table's length as the bound."""
    c = Tree(dev, store, (90, 0, 200), 40, 8, 4, 64, 16, seed=8)
    q, k, v = c.qkv()
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, scale=0.3)
    c.check(out, see=torch.tril(torch.ones(3, 40, 40)).bool(), scale=0.3)


@pytest.mark.parametrize("store", STORES)
def test_empty_rows_counts_and_shared_mask(dev, store):
    lens, t = (0, 70, 0, 33), 37
    c = Tree(dev, store, lens, t, 6, 2, 128, 16, seed=11)
    see = c.see[0].clone()
    see[5] = False
    see[36] = False
    see[:, 7] = False
    counts = [37, 20, 6, 0]
    out = torch.full((4, t, 6, 128), 5.0, dtype=c.dtype, device=dev)
    lse = torch.full((4, t, 6), 5.0, device=dev)
    q, k, v = c.qkv()
    ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), out=out, lse=lse, max_seq_len=70,
                       counts=torch.tensor(counts, dtype=torch.int32, device=dev))
    c.check(out, lse, see=see.expand(4, t, t), counts=counts)
    for b, n in enumerate(counts):
        assert torch.all(out[b, n:] == 5.0) and torch.all(lse[b, n:] == 5.0)
    assert torch.all(out[0, 5] == 0) and torch.all(lse[0, 36] == -math.inf)
    # counts and lengths outside their ranges are clamped
    wild = torch.tensor([99, -4, 6, 37], dtype=torch.int32, device=dev)
    long = torch.tensor([-3, 1 << 30, 0, 33], dtype=torch.int32, device=dev)
    got = ops.tree_attention(c.cache, long, q, k, v, mask=words_of(see).to(dev), counts=wild, max_seq_len=70,
                             out=torch.full_like(out, 5.0))
    c.check(got, see=see.expand(4, t, t), counts=[37, 0, 6, 37])
    assert torch.all(got[1] == 5.0)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_hidden_nodes_do_not_reach_a_row(dev, store, poison):
    """Nodes that hold NaN or infinities change the rows that see them, and no others."""
    c = Tree(dev, store, (50, 0), 70, 4, 2, 64, 16, seed=21)
    see = c.see.clone()
    see[:, :, 3] = False                                  # seen by nobody
    see[:, :, 40] = False
    see[:, 60:, 40] = True                                # seen by the last ten
    x = c.x.clone()
    x[:, 3, 4:] = poison                                  # key and value
    x[:, 40, 6:] = poison                                 # value
    q, k, v = c.qkv(x)
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), max_seq_len=50)
    calm = c.x.clone()
    calm[:, 3, 4:] = 0
    calm[:, 40, 6:] = 0
    c.check(out[:, :60], see=see, counts=[60, 60], x=calm)
    got = out[:, 60:].float()
    assert (torch.isnan(got) if math.isnan(poison) else got == poison).all()
    assert torch.isfinite(out[:, :60].float()).all()
    # the last node's own query and key: only its row
    x = c.x.clone()
    x[:, 69, :6] = math.nan
    q, k, v = c.qkv(x)
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(c.see).to(dev), max_seq_len=50)
    assert torch.isnan(out[:, 69].float()).all() and torch.isfinite(out[:, :69].float()).all()


def test_strides_and_alignment(dev):
    """Projections of another width, heads that are not 16-byte aligned, outputs in another order."""
    c = Tree(dev, torch.bfloat16, (100, 33), 5, 6, 2, 64, 16, seed=31)
    mask = words_of(c.see).to(dev)
    q, k, v = c.qkv()
    ref = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=mask, max_seq_len=100)
    odd = torch.zeros(2 * 5 * 10 * 67 + 1, dtype=torch.bfloat16, device=dev)[1:].view(2, 5, 10, 67)[..., :64]
    odd.copy_(c.x.to(dev))
    out = torch.zeros(10, 6, 2, 64, dtype=torch.bfloat16, device=dev)[:, :, 0].view(2, 5, 6, 64)
    got = ops.tree_attention(c.cache, c.seq_lens, odd[:, :, :6], odd[:, :, 6:8], odd[:, :, 8:], mask=mask, out=out, max_seq_len=100)
    assert got.data_ptr() == out.data_ptr() and torch.equal(got, ref)
    f = Tree(dev, torch.float32, (100, 33), 5, 6, 2, 64, 16, seed=31)
    q, k, v = f.qkv()
    ref = ops.tree_attention(f.cache, f.seq_lens, q, k, v, mask=mask, max_seq_len=100)
    odd = torch.zeros(2 * 5 * 10 * 67 + 1, device=dev)[1:].view(2, 5, 10, 67)[..., :64]
    odd.copy_(f.x.to(dev))
    assert torch.equal(ops.tree_attention(f.cache, f.seq_lens, odd[:, :, :6], odd[:, :, 6:8], odd[:, :, 8:], mask=mask, max_seq_len=100), ref)


@pytest.mark.parametrize("store", [torch.bfloat16, torch.float8_e4m3fn])
def test_offsets_past_32_bits(dev, store):
    """Blocks more than 2^32 bytes apart."""
    nkv, hd, block = 2, 128, 16
    stride = (1 << 31) + 4096                             # elements between blocks
    big = torch.empty(3 * stride, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn) if store != torch.bfloat16 \
        else torch.empty(3 * stride, dtype=store, device=dev)
    k = torch.as_strided(big, (3, nkv, block * hd), (stride, 2 * block * hd, 1))
    v = torch.as_strided(big, (3, nkv, block * hd), (stride, 2 * block * hd, 1), block * hd)
    e = torch.full((3, nkv, 2, block), 127, dtype=torch.uint8, device=dev) if store != torch.bfloat16 else None
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device=dev)
    cache = ops.PagedCache(k, v, block, table, None if e is None else e[:, :, 0], None if e is None else e[:, :, 1])
    small = make_cache(dev, store, (45,), nkv, hd, block)
    gen = seeded(2)
    x = randn(gen, 45, 2 * nkv, hd, dtype=torch.bfloat16).to(dev)
    seq, pos = (t.to(dev) for t in tokens((45,)))
    q = randn(gen, 1, 6, 8, hd, dtype=torch.bfloat16).to(dev)
    n = torch.tensor([45], dtype=torch.int32, device=dev)
    got = []
    for c in (cache, small):
        ops.cache_write(c, seq, pos, x[:, :nkv], x[:, nkv:])
        got.append((ops.tree_attention(c, n, q, q[:, :, :nkv], q[:, :, nkv:2 * nkv]), *ops.cache_read(c, seq, pos)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


# ---------------------------------------------------------------- together

def serving_step(c, rot, mask, counts, src, seq, pos, starts):
    """What a server does per step: rotate the drafts' projections, verify the tree, write the accepted nodes."""
    q, k, v = c.qkv()
    b, t = q.shape[:2]
    at = (c.seq_lens[:, None] + starts).reshape(-1)
    q2, k2 = ops.rotary(rot, at, q.reshape(b * t, *q.shape[2:]), k.reshape(b * t, *k.shape[2:]))
    k2 = k2.view(b, t, *k.shape[2:])
    out = ops.tree_attention(c.cache, c.seq_lens, q2.view(q.shape), k2, v, mask=mask, counts=counts, max_seq_len=max(c.lens))
    ops.cache_write(c.cache, seq, pos, k2.flatten(0, 1), v.flatten(0, 1), src_rows=src)
    return out, *ops.cache_read(c.cache, seq, pos, torch.float32)


@pytest.mark.parametrize("store", STORES)
def test_a_serving_step_captured_and_replayed(dev, store):
    """Rotation, tree, writing and reading in one graph, replayed with eager calls between, against the eager results."""
    lens = (100, 7, 64)
    c = Tree(dev, store, [n + 16 for n in lens], 12, 8, 2, 64, 16, seed=41)
    c.seq_lens, c.lens = torch.tensor(lens, dtype=torch.int32, device=dev), [n + 16 for n in lens]
    rot = ops.make_rotary(64, rotary_dim=32)
    depth = torch.tensor([[int(r.sum()) - 1 for r in s] for s in c.see], dtype=torch.int32, device=dev)
    mask = words_of(c.see).to(dev)
    counts = torch.tensor([12, 5, 9], dtype=torch.int32, device=dev)
    src = torch.tensor([0, 3, 12, 14, 24], dtype=torch.int32, device=dev)
    seq = torch.tensor([0, 0, 1, 1, 2], dtype=torch.int32, device=dev)
    pos = torch.tensor([100, 101, 7, 8, 64], dtype=torch.int32, device=dev)
    run = lambda: serving_step(c, rot, mask, counts, src, seq, pos, depth)  # noqa: E731
    c.x = c.x.to(dev)                                     # (its place stays while a graph reads it)
    live = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):                                    # two graphs, each with its own workspace
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = run()
        graphs.append((g, outs))
    rows = torch.arange(12, device=dev) < counts[:, None]
    for i in range(3):
        for g, outs in graphs:
            for o in outs:
                o.fill_(math.nan)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0][rows], live[0][rows]), i
            assert torch.equal(outs[1], live[1]) and torch.equal(outs[2], live[2]), i
        again = run()
        assert torch.equal(again[0][rows], live[0][rows])


def test_another_stream(dev):
    """Calls on a stream of their own, as torch's current stream and as a raw handle."""
    c = Tree(dev, torch.bfloat16, (900, 20), 6, 8, 2, 128, 16, seed=51)
    q, k, v = c.qkv()
    mask = words_of(c.see).to(dev)
    ref = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=mask, max_seq_len=900)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=mask, max_seq_len=900)
    b = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=mask, max_seq_len=900, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(a, ref) and torch.equal(b, ref)


def test_the_probe_reads_what_was_written(dev):
    """A prompt's keys and values, rotated and written by the operators, under the classification
    forward, against the probe's oracle on the cache as it stands; then accepted drafts, and again."""
    from paper_2608_28099_amd import configs, inputs
    from tests import helpers as H
    w = configs.SMALL_BF16.replace(name="written", seq_len=("list", (40, 1, 33, 100, 500)), seed=77)
    lens = np.array([30, 0, 33, 97, 490], dtype=np.int32)
    kv = inputs.kv_cache(w, inputs.seq_lens(w), dev)
    params = inputs.params(w, dev)
    cache = ops.PagedCache.from_kv(kv)
    cache.k.fill_(math.nan)
    cache.v.fill_(math.nan)
    rot = ops.make_rotary(w.head_dim, base=w.rope_base)
    gen = seeded(6)
    probe = binding.Probe(w)
    written = np.zeros(5, dtype=np.int32)
    for now in (lens, np.array([40, 1, 33, 100, 500], dtype=np.int32)):
        seq, pos = tokens([int(a - b) for a, b in zip(now, written)], [int(b) for b in written])
        x = randn(gen, len(seq), 4, 128, dtype=torch.bfloat16).to(dev)
        ops.cache_write(cache, seq.to(dev), pos.to(dev), x[:, :2], x[:, 2:], rotary=rot)
        written = now
        kv.seq_lens.copy_(torch.from_numpy(now))
        got = probe.forward(kv, params).cpu().numpy()
        ref = np.stack([o["logits"] for o in H.oracle_outputs(w, kv, params, range(5))])
        H.check_logits(got, ref, "bf16", "written cache")
    probe.close()
