"""The cache operators at the ends of what they take."""
from __future__ import annotations

import math

import pytest
import torch

from oracle import cacheops as oracle
from paper_2608_28099_amd import binding, ops
from tests.test_gpu_ops import STORES, Tree, make_cache, randn, rotation_error, seeded, tokens, words_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()
    return torch.device("cuda:0")


@pytest.mark.parametrize("layout,dim,n", [("half", 64, (1 << 24) + 5), ("half", 34, (1 << 24) + 5),
                                          ("interleaved", 64, (1 << 26) - 1), ("half", 64, (1 << 26) - 1)])
def test_rotary_of_the_most_rows(dev, layout, dim, n):
    """From 2^24 rows on a launch of one dimension is full (four rows a workgroup: 2^26); in place, against
    calls of fewer rows and, at the end, the definition."""
    rot = ops.make_rotary(64, rotary_dim=dim, layout=layout)
    gen = torch.Generator(device=dev).manual_seed(dim)
    x = torch.randn((n, 1, 64), generator=gen, device=dev, dtype=torch.bfloat16)
    pos = torch.randint(-1, 5000, (n,), generator=gen, device=dev, dtype=torch.int32)
    last, last_pos = x[-300:].cpu(), pos[-300:].cpu()
    ref = x.clone()
    step = 1 << 22
    for i in range(0, n, step):
        ops.rotary(rot, pos[i:i + step], ref[i:i + step], out=ref[i:i + step])
    assert ops.rotary(rot, pos, x, out=x).data_ptr() == x.data_ptr()
    assert torch.equal(x, ref)
    theta, scale = oracle.frequencies(dim)
    live = last_pos >= 0
    want = oracle.rotate(last, last_pos, theta, scale, layout)
    got = x[-300:].cpu()
    assert rotation_error(got[live], last[live], want[live], theta, scale, layout, last_pos[live]) <= 1
    assert torch.equal(got[~live], last[~live])


class Ladder:
    """A call whose scores are sign * c * 2^power times the scale, exactly until the scale: queries are
    2^(power / 2) in one dim, keys c * sign times the rest there, c a whole number.  One token of every sequence, cached
    or the first node, has the best c, by 1 at least: the others' weights vanish, so the row is that token's value."""

    def __init__(self, dev, store, lens, nodes, group, hd, sign, power, best, bound=None):
        gen = seeded(nodes + power)
        nkv, dim = 2, 5
        self.dtype = torch.float32 if store == torch.float32 else torch.bfloat16
        nq = nkv * group
        self.cache = make_cache(dev, store, lens, nkv, hd, 16, seed=4, fill=math.nan)
        if bound is not None:  # a table (and so a plan) of longer sequences
            t = self.cache.block_table
            t = torch.cat([t, t[:, -1:].expand(-1, -(-bound // 16) - t.shape[1])], 1).contiguous()
            self.cache = ops.PagedCache(self.cache.k, self.cache.v, 16, t, self.cache.k_exponents, self.cache.v_exponents)
        seq, pos = tokens(lens)
        c = torch.randint(2, 4, (len(seq),), generator=gen).double()
        cn = torch.randint(2, 4, (len(lens), nodes), generator=gen).double()
        top = 1.0 if sign < 0 else 4.0
        winner = torch.tensor([2 * n // 3 for n in lens])
        first = torch.tensor([sum(lens[:b]) for b in range(len(lens))])
        if best == "cached":
            c[first + winner] = top
        else:
            cn[:, 0] = top
        kv = torch.randn((len(seq), 2 * nkv, hd), generator=gen).double()
        kv[:, :nkv] = 0
        kv[:, :nkv, dim] = (sign * c * 2.0 ** (power - power // 2))[:, None]
        kv = kv.to(self.dtype).to(dev)
        ops.cache_write(self.cache, seq.to(dev), pos.to(dev), kv[:, :nkv], kv[:, nkv:])
        q = torch.zeros((len(lens), nodes, nq, hd), dtype=torch.float64)
        q[..., dim] = 2.0 ** (power // 2)
        k = torch.zeros((len(lens), nodes, nkv, hd), dtype=torch.float64)
        k[..., dim] = (sign * cn * 2.0 ** (power - power // 2))[..., None]
        v = torch.randn((len(lens), nodes, nkv, hd), generator=gen)
        self.q, self.k, self.v = (x.to(self.dtype).to(dev) for x in (q, k, v))
        if best == "cached":
            value = ops.cache_read(self.cache, torch.arange(len(lens), dtype=torch.int32, device=dev),
                                   winner.int().to(dev), torch.float32)[1].cpu()
        else:
            value = self.v[:, 0].float().cpu()
        self.value = value[:, None, :, None].expand(-1, nodes, -1, group, -1).reshape(len(lens), nodes, nq, hd).double()
        self.score = sign * top * 2.0 ** power
        self.seq_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
        self.bound = max(lens) if bound is None else bound

    def check(self, scale):
        lse = torch.zeros(self.q.shape[:3], device=self.q.device)
        out = ops.tree_attention(self.cache, self.seq_lens, self.q, self.k, self.v, lse=lse, scale=scale,
                                 max_seq_len=self.bound).cpu().double()
        # one weight, within a factor of 2^8 of 1: rounded (bf16), its product and the sum over it; the result's rounding
        u = 0.0 if self.dtype == torch.float32 else 2.0 ** -8
        tol = (2 * u + 2.0 ** -21) * self.value.abs()
        assert torch.isfinite(out).all(), "not finite"
        assert torch.all((out - self.value).abs() <= tol), float(((out - self.value).abs() - tol).max())
        # the scale and its product with log2(e), the score, the maximum times ln(2): half a step each, two spare
        want = self.score * scale
        assert torch.all((lse.cpu().double() - want).abs() <= 6 * 2.0 ** -24 * abs(want) + 2.0 ** -20), (float(lse.flatten()[0]), want)


# sequences, nodes, query heads per KV head, the bound that plans the call: one split and several; fp32 by eight waves
# and staged; waves of 16 rows and, from 129 rows with much to do, of 32
LADDERS = [((40, 7), 3, 1, None), ((3000, 700), 5, 4, None), ((300, 90), 40, 5, None), ((300, 90), 40, 5, 131072)]


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lens,nodes,group,bound", LADDERS)
@pytest.mark.parametrize("best", ["cached", "node"])
@pytest.mark.parametrize("power", [101, 120])
def test_scores_far_below_zero(dev, store, lens, nodes, group, bound, best, power):
    """Rows all of whose scores are below -1e30 see their tokens all the same.  (The scale is ln 2, which leaves whole
    scores in the kernels' units.)"""
    Ladder(dev, store, lens, nodes, group, 64, -1, power, best, bound).check(math.log(2.0))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lens,nodes,group,bound", LADDERS)
@pytest.mark.parametrize("best", ["cached", "node"])
@pytest.mark.parametrize("sign,power", [(1, 26), (-1, 26), (1, 31), (-1, 33), (1, 36), (-1, 45), (1, 100), (-1, 118)])
def test_scores_whose_steps_are_large(dev, store, lens, nodes, group, bound, best, sign, power):
    """Scores so large that one step of fp32 between them is many powers of two of the weights."""
    for scale in (0.125, 0.3):
        Ladder(dev, store, lens, nodes, group, 64, sign, power, best, bound).check(scale)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lens,group,bound", [((50, 0), 2, None), ((300, 90), 5, None), ((300, 90), 5, 131072)])
@pytest.mark.parametrize("poison", [math.nan, math.inf, -math.inf])
def test_values_that_are_not_finite_under_weights_that_vanish(dev, store, lens, group, bound, poison):
    """A node's value reaches every row that sees it, as a cached one does, also where its weight is too small
    for fp32 (0 times infinity or NaN is NaN); rows that do not see it stay as they are."""
    t, nq, nkv, hd = 40, 2 * group, 2, 64
    c = Tree(dev, store, lens, t, nq, nkv, hd, 16, seed=22)
    if bound is not None:
        table = c.cache.block_table
        table = torch.cat([table, table[:, -1:].expand(-1, -(-bound // 16) - table.shape[1])], 1).contiguous()
        c.cache = ops.PagedCache(c.cache.k, c.cache.v, 16, table, c.cache.k_exponents, c.cache.v_exponents)
    see = torch.eye(t).bool().expand(len(lens), t, t).clone()
    see[:, 20:, 7] = True
    x = c.x.clone()
    x[:, :, :nq, 0] = 64.0                                # node 7's scores: near -64 * 512 / 8 in the rows that see it
    x[:, 7, nq:nq + nkv, 0] = -512.0
    x[:, 7, nq + nkv:] = poison
    q, k, v = c.qkv(x)
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), max_seq_len=bound or max(lens)).cpu()
    assert not torch.isfinite(out[:, 20:].float()).any()
    assert torch.isfinite(out[:, :7].float()).all() and torch.isfinite(out[:, 8:20].float()).all()


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("hd", [64, 128])
def test_the_largest_blocks(dev, store, hd):
    """A head's block of 2^31 bytes, one per sequence: a token near its end and one in the middle are found."""
    size = torch.empty(0, dtype=store).element_size()
    n = (1 << 31) // (hd * size)
    dtype = torch.float32 if store == torch.float32 else torch.bfloat16
    cache = ops.PagedCache.allocate(store, 2, 1, hd, n, batch=2, device=dev)
    pos = torch.tensor([n - 2, n // 2 + 7], dtype=torch.int32, device=dev)
    seq = torch.tensor([0, 1], dtype=torch.int32, device=dev)
    x = randn(seeded(hd), 2, 2, hd).to(dtype).to(dev)
    x[:, 0] = 16.0
    ops.cache_write(cache, seq, pos, x[:, :1], x[:, 1:])
    q = torch.full((2, 1, 4, hd), 16.0, dtype=dtype, device=dev)
    zero = torch.zeros((2, 1, 1, hd), dtype=dtype, device=dev)
    got = ops.tree_attention(cache, torch.tensor([n - 1, n], dtype=torch.int32, device=dev), q, zero, zero, scale=1.0)
    value = ops.cache_read(cache, seq, pos, dtype)[1]
    # scores of 0 and of 16 * 16 * hd >= 16384: the weights of all others vanish
    assert torch.equal(got, value[:, None].expand(-1, -1, 4, -1))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("largest", [1.0, 224.0, 240.0, 255.0, 256.0, 448.0])
def test_single_query_values_over_8_bit_keys(dev, hd, largest):
    """One query value alone decides each score (keys of one value): off by 2^-14 / 224 of its row's largest at most, and
    exact from 2^-6 / 224 of it on."""
    gen = seeded(int(largest))
    n = 60
    q = torch.randint(128, 256, (n,), generator=gen).double() * torch.exp2(-7.0 - torch.arange(n) % 24) * 2.0 ** 8
    q[0] = 241 * 2.0 ** -14
    q = torch.where(q > largest, q * 2.0 ** -9, q)
    cache = make_cache(dev, torch.float8_e4m3fn, (1,), 1, hd, 16, fill=math.nan)
    kv = torch.zeros((1, 2, hd))
    kv[:, 0, 9] = 1.0
    kv[:, 1] = 1.0
    ids = torch.zeros(1, dtype=torch.int32, device=dev)
    ops.cache_write(cache, ids, ids, kv[:, :1].to(dev), kv[:, 1:].to(dev))
    x = torch.zeros((1, n, 1, hd))
    x[0, :, 0, 9] = q
    x[0, :, 0, 40] = largest
    x = x.bfloat16().to(dev)
    lse = torch.zeros((1, n, 1), device=dev)
    ops.tree_attention(cache, torch.ones(1, dtype=torch.int32, device=dev), x, x, x, lse=lse, scale=1.0, max_seq_len=1,
                       mask=torch.zeros((n, 2), dtype=torch.int32, device=dev))
    off = (lse[0, :, 0].cpu().double() - q).abs()
    exact = 4 * 2.0 ** -24 * q                            # the factor log2(e), its product, ln(2) and that product
    assert torch.all(off <= exact + 2.0 ** -14 / 224 * largest), float(off.max())
    assert torch.all((off <= exact)[q >= 2.0 ** -6 / 224 * largest])
