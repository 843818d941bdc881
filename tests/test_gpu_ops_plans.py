"""Tree attention over the launch plans that small calls do not reach: splits of many windows of
block ids, more splits than one round of the join, more sequences than the work items' scan
takes, contiguous storage; and seeded random shapes of all the cache operators."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2608_28099_amd import binding, ops
from tests.test_gpu_ops import STORES, Tree, make_cache, seeded, tokens, words_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    binding.load()
    return torch.device("cuda:0")


def run(c, **kw):
    q, k, v = c.qkv()
    lse = torch.zeros((len(c.lens), c.t, c.nq), device=c.dev)
    out = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(c.see).to(c.dev), lse=lse,
                             max_seq_len=max(c.lens), **kw)
    return out, lse


@pytest.mark.parametrize("store", [torch.bfloat16, torch.float8_e4m3fn])
@pytest.mark.parametrize("contiguous", [False, True])
def test_splits_of_more_block_ids_than_are_held_at_once(dev, store, contiguous):
    """131072 tokens in blocks of 16, splits of 16384 (1024 ids, four windows of 256)."""
    lens = (131072, 40) if contiguous else (131072, 40, 3, 17000, 0, 9, 1, 64, 5, 7, 8, 2)
    nkv = 48 if contiguous else 8
    c = Tree(dev, store, lens, 1, nkv, nkv, 64, 16, seed=61, contiguous=contiguous)
    out, lse = run(c)
    # every sequence but the longest whole, of the longest the first and last heads
    c.check(out, lse, sequences=range(1, len(lens)))
    from oracle import cacheops as oracle
    from tests.test_gpu_ops import dense
    kc, vc = dense(c.cache, 0, lens[0])
    for g in (0, nkv - 1):
        x = c.x[0]
        ref, rl, mag, big = oracle.tree_attention(x[:, g:g + 1], kc[g:g + 1], vc[g:g + 1], x[:, nkv + g:nkv + g + 1],
                                                  x[:, 2 * nkv + g:2 * nkv + g + 1], c.see[0])
        # as Tree.check: a weight's rounding, the result's, the scores', and sums of n terms (in splits of 16384,
        # eight of which are joined)
        eps = 2 * (64 * 2.0 ** -24 * big + 2.0 ** -22) + 2 * 16400 * 2.0 ** -24
        tol = mag * (2.0 ** -8 + eps) + 2.0 ** -8 * ref.abs()
        assert torch.all((out[0, :, g:g + 1].cpu().double() - ref).abs() <= tol)
        assert torch.all((lse[0, :, g:g + 1].cpu().double() - rl).abs() <= eps + 2.0 ** -22 * (1 + rl.abs()))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("hd,nodes", [(64, 3), (128, 20)])
def test_more_splits_than_one_round_of_the_join(dev, store, hd, nodes):
    """One sequence of 20000 tokens, two KV heads: about 79 splits of 256."""
    c = Tree(dev, store, (20000,), nodes, 4, 2, hd, 16, seed=62)
    c.check(*run(c))


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("batch", [64, 65, 1024, 1100])
def test_many_sequences(dev, store, batch):
    """Around the 64 sequences that one step of the work items' scan takes and the 1024 that it takes at all;
    lengths of several splits among many short ones."""
    gen = seeded(batch)
    lens = [int(x) for x in torch.randint(0, 40, (batch,), generator=gen)]
    for b in (0, 1, 63, batch // 2, batch - 1):
        lens[b] = 4100 + b
    lens[5] = 2048 if batch > 100 else 2049
    c = Tree(dev, store, lens, 2, 2, 1, 64, 16, seed=63)
    out, lse = run(c)
    c.check(out, lse, sequences=[0, 1, 2, 5, 62, 63, 64 % batch, batch // 2, batch - 2, batch - 1])
    # and every sequence against calls of its own size
    again = ops.tree_attention(c.cache, c.seq_lens, *c.qkv(), mask=words_of(c.see).to(dev), max_seq_len=c.cache.capacity)
    assert torch.allclose(out.float(), again.float(), rtol=2.0 ** -6, atol=1e-4)


@pytest.mark.parametrize("store", STORES)
def test_the_same_call_under_two_bounds_of_the_length(dev, store):
    """Splits change with max_seq_len, results only by roundings; a bound below a length clamps it."""
    c = Tree(dev, store, (3000, 700, 0), 5, 8, 2, 128, 16, seed=64)
    a, _ = run(c)
    q, k, v = c.qkv()
    m = words_of(c.see).to(dev)
    b = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=m)
    assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -6, atol=1e-4)
    short = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=m, max_seq_len=700)
    same = ops.tree_attention(c.cache, torch.clamp(c.seq_lens, max=700), q, k, v, mask=m, max_seq_len=700)
    assert torch.equal(short, same)


def test_two_streams_and_a_workspace_of_the_callers(dev):
    """Overlapping calls with memory of their own, and one after the other on one workspace full of NaN."""
    c = Tree(dev, torch.bfloat16, (5000, 900), 17, 8, 2, 128, 16, seed=65)
    ref, _ = run(c)
    q, k, v = c.qkv()
    m = words_of(c.see).to(dev)
    call = lambda **kw: ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=m, max_seq_len=5000, **kw)  # noqa: E731
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            outs.append(call())
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for o in outs)
    n = ops.tree_workspace_bytes(c.cache, 8, torch.bfloat16, 17, max_seq_len=5000)
    ws = torch.empty(n, dtype=torch.uint8, device=dev)
    ws.view(torch.float32).fill_(math.nan)
    assert torch.equal(call(workspace=ws), ref) and torch.equal(call(workspace=ws), ref)
    with pytest.raises(binding.ProbeError):
        call(workspace=ws[:n - 256])
    # a workspace for larger calls serves smaller ones
    n2 = ops.tree_workspace_bytes(c.cache, 8, torch.bfloat16, 256)
    assert n2 >= n and torch.equal(call(workspace=torch.empty(n2, dtype=torch.uint8, device=dev)), ref)


@pytest.mark.parametrize("seed", range(24))
def test_random_trees(dev, seed):
    gen = seeded(1000 + seed)
    pick = lambda *xs: xs[int(torch.randint(0, len(xs), (1,), generator=gen))]  # noqa: E731
    hd, nkv, group = pick(64, 128), pick(1, 2, 3), pick(1, 2, 4, 5, 7)
    t, block, batch = pick(1, 2, 7, 16, 31, 33, 65), pick(16, 32, 64, 128), pick(1, 2, 5)
    hi = pick(1, 40, 300, 2500)
    lens = [int(x) for x in torch.randint(0, hi + 1, (batch,), generator=gen)]
    store = pick(*STORES)
    print(f"[tree] seed {seed}: {store} lens {lens} nodes {t} heads {nkv}x{group} hd {hd} block {block}", flush=True)
    c = Tree(dev, store, lens, t, nkv * group, nkv, hd, block, seed=seed, contiguous=pick(False, False, True))
    see = c.see & (torch.rand(c.see.shape, generator=gen) < pick(1.0, 0.6))
    counts = [int(x) for x in torch.randint(0, t + 1, (batch,), generator=gen)]
    q, k, v = c.qkv()
    out = torch.full(q.shape, 3.0, dtype=c.dtype, device=dev)
    lse = torch.full(q.shape[:3], 3.0, device=dev)
    ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), out=out, lse=lse,
                       counts=torch.tensor(counts, dtype=torch.int32, device=dev))
    c.check(out, lse, see=see, counts=counts)
    for b, n in enumerate(counts):
        assert torch.all(out[b, n:] == 3.0) and torch.all(lse[b, n:] == 3.0)


@pytest.mark.parametrize("seed", range(12))
def test_random_rows_in_and_out_of_a_cache(dev, seed):
    """Rows of several sequences in runs that start anywhere, some reversed, some scattered."""
    gen = seeded(2000 + seed)
    pick = lambda *xs: xs[int(torch.randint(0, len(xs), (1,), generator=gen))]  # noqa: E731
    store, dtype = pick(*STORES), pick(torch.float32, torch.bfloat16)
    hd, nkv, block = pick(64, 128), pick(1, 2, 5), pick(16, 32, 128)
    starts = [int(x) for x in torch.randint(0, 70, (4,), generator=gen)]
    lens = [int(x) for x in torch.randint(0, 150, (4,), generator=gen)]
    print(f"[rows] seed {seed}: {store} {dtype} hd {hd} block {block} starts {starts} lens {lens}", flush=True)
    cache = make_cache(dev, store, [a + b for a, b in zip(starts, lens)], nkv, hd, block, seed)
    seq, pos = tokens(lens, starts)
    n = len(seq)
    order = torch.arange(n)
    if seed % 3 == 1:
        order = order.flip(0)
    if seed % 3 == 2 and n > 40:
        order[20:40] = order[20:40][torch.randperm(20, generator=gen)]
    seq, pos = seq[order].to(dev), pos[order].to(dev)
    x = torch.randn((n, 2 * nkv, hd), generator=gen).to(dtype).to(dev)
    if n:
        ops.cache_write(cache, seq, pos, x[:, :nkv], x[:, nkv:])
    k, v = ops.cache_read(cache, seq, pos, torch.float32)
    if store == torch.float8_e4m3fn:
        from oracle import cacheops as oracle
        for got, want in ((k, x[:, :nkv]), (v, x[:, nkv:])):
            val, byte = oracle.quantise(want.cpu())
            assert torch.equal(got.cpu().double(), val * torch.exp2(byte.double() - 127)[..., None])
    else:
        assert torch.equal(k, x[:, :nkv].to(store).float()) and torch.equal(v, x[:, nkv:].to(store).float())


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("hd,nodes,nq,nkv", [(128, 64, 8, 2), (128, 43, 12, 2), (64, 256, 3, 3), (64, 33, 32, 4), (128, 3, 64, 1)])
@pytest.mark.parametrize("cut", [False, True])
@pytest.mark.parametrize("much", [False, True])
def test_many_query_rows(dev, store, hd, nodes, nq, nkv, cut, much):
    """192 rows and more per KV head, whole groups and partly filled ones, sequences of one split and of several,
    masks that leave rows empty, nodes that are not finite; planned for the lengths at hand (waves of 16 rows), and for
    as many tokens as waves of 32 rows take."""
    lens = (0, 1, 33, 47, 64, 1000, 2700) if cut else (700, 13)
    c = Tree(dev, store, lens, nodes, nq, nkv, hd, 16, seed=66 + nodes)
    batch, gen = len(lens), seeded(67)
    bound = max(lens)
    if much:
        groups = -(-nodes * nq // nkv // 128)
        bound = max(bound, 256 * -(-6 * 256 // (nkv * batch * groups)))
        table = c.cache.block_table
        table = torch.cat([table, table[:, -1:].expand(-1, -(-bound // 16) - table.shape[1])], 1).contiguous()
        c.cache = ops.PagedCache(c.cache.k, c.cache.v, 16, table, c.cache.k_exponents, c.cache.v_exponents)
    see = c.see & (torch.rand(c.see.shape, generator=gen) < 0.7)
    see[:, :, nodes // 2] = False
    x, calm = c.x.clone(), c.x.clone()
    x[:, nodes // 2, nq:] = math.nan  # seen by nobody
    calm[:, nodes // 2, nq:] = 0
    counts = [int(n) for n in torch.randint(1, nodes + 1, (batch,), generator=gen)] if cut else [nodes] * batch
    q, k, v = c.qkv(x)
    out = torch.full(q.shape, 3.0, dtype=c.dtype, device=dev)
    lse = torch.full(q.shape[:3], 3.0, device=dev)
    ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), out=out, lse=lse,
                       counts=torch.tensor(counts, dtype=torch.int32, device=dev), max_seq_len=bound)
    c.check(out, lse, see=see, counts=counts, x=calm)
    for b, n in enumerate(counts):
        assert torch.all(out[b, n:] == 3.0) and torch.all(lse[b, n:] == 3.0)
    # infinite values reach the rows that see them, and those rows only
    see[:, :, nodes // 2] = torch.rand((batch, nodes), generator=gen) < 0.5
    x = c.x.clone()
    x[:, nodes // 2, nq + nkv:] = math.inf
    q, k, v = c.qkv(x)
    got = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=words_of(see).to(dev), max_seq_len=bound).cpu()
    hit = see[:, :, nodes // 2].clone()
    assert torch.all(got[hit].float() == math.inf)
    see[:, :, nodes // 2] = False
    rest = ops.tree_attention(c.cache, c.seq_lens, *c.qkv(), mask=words_of(see).to(dev), max_seq_len=bound).cpu()
    # (to the tolerance, not to the bit: rows of a wave move their reference maximum together, so what one of them sees
    # can change at which power of two another's weights are rounded)
    c.check(torch.where(hit[:, :, None, None], rest, got), see=see)


@pytest.mark.parametrize("store", STORES)
def test_single_nodes_of_packed_projections(dev, store):
    c = Tree(dev, store, (300, 0, 17), 1, 8, 2, 128, 16, seed=68)
    ref = ops.tree_attention(c.cache, c.seq_lens, *c.qkv(), max_seq_len=300)
    packed = c.x[:, 0].to(dev)  # [batch, heads, hd]
    q, k, v = (x.unsqueeze(1) for x in packed.split([8, 2, 2], 1))
    assert torch.equal(ops.tree_attention(c.cache, c.seq_lens, q, k, v, max_seq_len=300), ref)


def test_results_on_a_given_stream_use_that_streams_memory(dev):
    """Memory that the current stream still reads (freed, but its work is pending) is not written by a call on
    another stream; results outlive the call's own references."""
    side = torch.cuda.Stream()
    rot = ops.make_rotary(128)
    q = torch.randn(4096, 8, 128, device=dev)
    pos = torch.arange(4096, dtype=torch.int32, device=dev)
    ref = ops.rotary(rot, pos, q)
    torch.cuda.synchronize()
    a = torch.full(q.shape, 2.0, device=dev)
    b = torch.randn(4096, 4096, device=dev)
    torch.cuda.synchronize()
    for _ in range(20):  # some milliseconds before the sum below
        b = torch.mm(b, b).clamp_(-1, 1)
    total = a.sum(dtype=torch.float64)
    at = a.data_ptr()
    del a
    y = ops.rotary(rot, pos, q, stream=side.cuda_stream)
    assert y.data_ptr() != at
    torch.cuda.synchronize()
    assert float(total) == 2.0 * q.numel() and torch.equal(y, ref)


@pytest.mark.parametrize("store", STORES)
def test_calls_without_rows(dev, store):
    dtype = torch.float32 if store == torch.float32 else torch.bfloat16
    cache = make_cache(dev, store, (20, 5), 2, 64, 16, fill=1.0)
    before = [t.clone() for t in (cache.k, cache.v)]
    none = torch.empty(0, dtype=torch.int32, device=dev)
    x = torch.empty((0, 2, 64), dtype=dtype, device=dev)
    rot = ops.make_rotary(64)
    assert ops.rotary(rot, none, x).shape == x.shape
    assert [t.shape for t in ops.rotary(rot, none, x, x)] == [x.shape, x.shape]
    ops.cache_write(cache, none, none, x, x)
    ops.cache_write(cache, none, none, torch.ones((3, 2, 64), dtype=dtype, device=dev), torch.ones((3, 2, 64), dtype=dtype, device=dev),
                    src_rows=none, rotary=rot)
    ids = torch.zeros(3, dtype=torch.int32, device=dev)
    ops.cache_write(cache, ids, ids, x, x, src_rows=ids)   # no row to take: nothing is written
    assert ops.cache_read(cache, none, none, dtype)[0].shape == x.shape
    for a, b in zip(before, (cache.k, cache.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    empty = ops.PagedCache(cache.k, cache.v, 16, torch.empty((0, 4), dtype=torch.int32, device=dev), cache.k_exponents, cache.v_exponents)
    q = torch.empty((0, 3, 4, 64), dtype=dtype, device=dev)
    assert ops.tree_attention(empty, none, q, q[:, :, :2], q[:, :, :2]).shape == q.shape


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("which", ["k", "v"])
def test_one_side_read_into_padded_rows(dev, store, which):
    """Keys or values alone, into rows that are not 16-byte aligned, some tokens several times, some rows skipped."""
    gen = seeded(70)
    cache = make_cache(dev, store, (90, 33), 3, 64, 16, 1)
    seq, pos = tokens((90, 33))
    x = torch.randn((len(seq), 6, 64), generator=gen).to(dev)
    ops.cache_write(cache, seq.to(dev), pos.to(dev), x[:, :3], x[:, 3:])
    order = torch.cat([torch.arange(60), torch.tensor([5, 5, 5, 122, 0]), torch.arange(20, 60)])
    s, p = seq[order].to(dev), pos[order].to(dev)
    s[7], p[9] = -1, 1 << 30
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.full((len(order), 3, 67), 7.0, dtype=dtype, device=dev)
        got = ops.cache_read(cache, s, p, **{which: out[..., :64]})
        assert got[0 if which == "k" else 1].data_ptr() == out.data_ptr() and got[1 if which == "k" else 0] is None
        whole = ops.cache_read(cache, seq.to(dev), pos.to(dev), dtype)[0 if which == "k" else 1][order.to(dev)]
        live = torch.ones(len(order), dtype=torch.bool)
        live[7] = live[9] = False
        assert torch.equal(out[live][..., :64], whole[live]) and torch.all(out[~live] == 7.0) and torch.all(out[..., 64:] == 7.0)


@pytest.mark.parametrize("store", STORES)
@pytest.mark.parametrize("lens,t,nq,nkv,hd,block", [
    ((300, 7), 256, 32, 1, 64, 16),        # 8192 query rows
    ((20,), 1, 4096, 4096, 64, 16),        # the most heads
    ((20, 0), 3, 4096, 2, 64, 16),         # 2048 heads on one
    ((5000, 1, 4096), 9, 4, 2, 128, 4096)])
def test_sizes_at_their_limits(dev, store, lens, t, nq, nkv, hd, block):
    c = Tree(dev, store, lens, t, nq, nkv, hd, block, seed=71)
    c.check(*run(c))


def test_calls_from_several_threads(dev):
    import threading
    c = Tree(dev, torch.bfloat16, (600, 31), 9, 8, 2, 128, 16, seed=72)
    ref, _ = run(c)
    q, k, v = c.qkv()
    mask = words_of(c.see).to(dev)
    rot = ops.make_rotary(128)
    pos = torch.arange(18, dtype=torch.int32, device=dev)
    turned = ops.rotary(rot, pos, q.reshape(18, 8, 128))
    torch.cuda.synchronize()
    bad = []

    def work():
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            for _ in range(20):
                a = ops.tree_attention(c.cache, c.seq_lens, q, k, v, mask=mask, max_seq_len=600)
                b = ops.rotary(rot, pos, q.reshape(18, 8, 128))
                side.synchronize()
                if not (torch.equal(a, ref) and torch.equal(b, turned)):
                    bad.append(1)

    threads = [threading.Thread(target=work) for _ in range(3)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not bad


def test_refusals_of_tensors(dev):
    rot = ops.make_rotary(64)
    x = torch.zeros((2, 3, 64), device=dev)
    pos = torch.zeros(2, dtype=torch.int32, device=dev)
    for args, kw in (((rot, pos.long(), x), {}), ((rot, pos, x.half()), {}), ((rot, pos, x[..., ::2]), {}), ((rot, pos.cpu(), x), {}),
                     ((rot, pos, x), dict(k_out=x)), ((rot, pos, x), dict(out=x[:1])), ((rot, pos[:1], x), {})):
        with pytest.raises(ValueError):
            ops.rotary(*args, **kw)
    c = Tree(dev, torch.bfloat16, (20, 3), 4, 4, 2, 64, 16)
    q, k, v = c.qkv()
    for kw in (dict(seq_lens=c.seq_lens[:1]), dict(q=q[:1]), dict(k=k[:, :, :1]), dict(scale=-1.0), dict(scale=math.inf), dict(scale=0.0),
               dict(mask=torch.zeros((2, 3, 1), dtype=torch.int32, device=dev)), dict(lse=torch.zeros(2, 4, 4)),
               dict(workspace=torch.zeros(64, device=dev)), dict(counts=torch.zeros(3, dtype=torch.int32, device=dev))):
        a = dict(dict(cache=c.cache, seq_lens=c.seq_lens, q=q, k=k, v=v), **kw)
        with pytest.raises(ValueError):
            ops.tree_attention(**a)
    for kw in (dict(max_seq_len=c.cache.capacity + 1), dict(max_seq_len=-1), dict(workspace=torch.zeros(16, dtype=torch.uint8, device=dev))):
        with pytest.raises(binding.ProbeError):
            ops.tree_attention(c.cache, c.seq_lens, q, k, v, **kw)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("power", [0, 100, -100])
def test_queries_of_wide_range_over_8_bit_keys(dev, hd, power):
    """Queries from 2^-40 to 4 in a row, rows of zeros, of one value, and whole calls times a large or small power of two
    (and the scale over it)."""
    from oracle import cacheops as oracle
    from tests.test_gpu_ops import dense
    lens, t, nq, nkv = (130, 700), 9, 4, 2
    c = Tree(dev, torch.float8_e4m3fn, lens, t, nq, nkv, hd, 16, seed=73)
    gen = seeded(74)
    x = c.x.float()
    small = torch.exp2(-40 * torch.rand(x[:, :, :nq].shape, generator=gen))
    x[:, 1:5, :nq] *= small[:, 1:5]
    x[:, 5, :nq] = 0
    x[:, 6, :nq] = 0
    x[:, 6, :nq, 7] = 3.0
    x = (x * 3).bfloat16()
    scale = hd ** -0.5
    q, k, v = c.qkv(x)
    got = ops.tree_attention(c.cache, c.seq_lens, q * 2.0 ** power, k, v, mask=words_of(c.see).to(dev), max_seq_len=700,
                             scale=scale * 2.0 ** -power).cpu()
    for b, n in enumerate(lens):
        kc, vc = dense(c.cache, b, n)
        q, k, v = x[b, :, :nq], x[b, :, nq:nq + nkv], x[b, :, nq + nkv:]
        ref, _, mag, big = oracle.tree_attention(q, kc, vc, k, v, c.see[b], scale)
        # Tree.check's terms, and each query value off by 2^-22 of its row's largest
        far = scale * 2.0 ** -22 * q.double().abs().amax(-1, keepdim=True) * kc.double().abs().sum(-1).max()
        eps = 2 * (hd * 2.0 ** -24 * big + 2.0 ** -22) + 2 * (n + t + 8) * 2.0 ** -24
        eps = eps + 2 * (far if torch.as_tensor(big).dim() == 3 else far.max())
        tol = mag * (2.0 ** -8 + eps) * (1 + 2.0 ** -6) + 2.0 ** -8 * ref.abs() + 1e-30
        assert torch.all((got[b].double() - ref).abs() <= tol), float(((got[b].double() - ref).abs() / tol).max())
