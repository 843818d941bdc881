"""Performance cases of the operators around a speculative head's paged cache.

A server that drafts with the head and probes with it does four things on one cache:

  rotary  rotate the rows of the query and key projections at their positions (whole
          head or its first dims, half or interleaved pairs, frequencies scaled for long
          contexts); transposed, the gradient's rotation
  write   put rows of keys and values into their slots of the paged cache, rotated on
          the way if asked, as bf16, fp32 or 8-bit values with one exponent per token
          and head, and read those rows back
  read    gather tokens of a cache into rows
  tree    attention of a tree of drafted tokens over the cache and the drafted tokens
          that the tree's mask shows to each; one node is plain decoding

Head shapes, batches and context lengths are those of paper_2608_28099_amd.configs (tiny,
small, 4B-, 9B- and 27B-shaped heads, the long context).  Where ``own`` is true ``run``
makes the library's calls, else it computes the same in elementary torch operations.
Lengths and trees belong to the case; every value and block placement comes from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# query heads, KV heads, head dim
HEADS = {
    "tiny": (4, 2, 64),         # configs.TINY_F32
    "small": (8, 2, 128),       # configs.SMALL_BF16
    "small_g5": (10, 2, 128),   # configs.SMALL_G5_BF16
    "4b": (32, 8, 128),         # configs.QWEN4B_BF16, QWEN9B_BF16
    "27b": (40, 8, 128),        # configs.QWEN27B_BF16
}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def _rot(dim, layout="half", scaling="none", factor=1.0, original=0, base=10000.0):
    return {"dim": dim, "layout": layout, "scaling": scaling, "factor": factor, "original": original, "base": base}


def _rotary(name, head, rows, far, rot, dtype="bf16", transpose=False):
    """rows: rows of projections; far: the positions' upper end."""
    c = {"op": "rotary", "head": head, "rows": rows, "far": far, "dtype": dtype, "transpose": transpose,
         **{"rot_" + k: v for k, v in rot.items()}}
    return dict(c, name=name) if name else c


def _cache(name, op, head, batch, lo, hi, start, cache, dtype, rot=None, pick=0, block=16):
    """write, read: lo..hi rows for each sequence, after up to `start` tokens that are there;
    pick: the rows are some of the pick nodes of each sequence's tree (0: all rows in order)."""
    c = {"op": op, "head": head, "batch": batch, "lo": lo, "hi": hi, "start": start, "cache": cache, "dtype": dtype,
         "pick": pick, "block": block, "rotated": rot is not None,
         **{"rot_" + k: v for k, v in (rot or _rot(0)).items()}}
    return dict(c, name=name) if name else c


def _tree(name, head, batch, nodes, lo, hi, cache, dtype="bf16", block=16, ragged=False, empty=False, lse=False):
    """lo..hi: cached tokens; ragged: sequences with fewer nodes; empty: nodes that see no node, not even themselves."""
    c = {"op": "tree", "head": head, "batch": batch, "nodes": nodes, "lo": lo, "hi": hi, "cache": cache, "dtype": dtype,
         "block": block, "ragged": ragged, "empty": empty, "lse": lse}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the soft rows of the smallest head, interleaved pairs: the smallest call there is
        _rotary("rotary_tiny_f32", "tiny", 16, 260, _rot(64, "interleaved"), dtype="f32"),
        # one decoding step of 128 requests far past the trained length
        _rotary("rotary_decode_yarn", "4b", 128, 131072, _rot(128, scaling="yarn", factor=4.0, original=32768)),
        # the gradient of a training batch's projections, half of each head rotated
        _rotary("rotary_grad_partial", "27b", 16384, 32768, _rot(64, scaling="linear", factor=2.0), transpose=True),
        # the accepted nodes of 128 requests' trees enter a bf16 cache
        _cache("write_accepted", "write", "4b", 128, 1, 6, 8192, "bf16", "f32", pick=16),
        # prompts of 2K-4K tokens rotated, quantised, written and read back
        _cache("write_prompts_e4m3", "write", "4b", 16, 2048, 4096, 0, "e4m3", "bf16", rot=_rot(128)),
        # prefixes of 32 requests gathered from an 8-bit cache
        _cache("read_prefix_e4m3", "read", "4b", 32, 1024, 4096, 0, "e4m3", "bf16"),
        # a small tree over the fp32 head's configured cache
        _tree("tree_tiny_f32", "tiny", 4, 4, 256, 256, "f32", dtype="f32", lse=True),
        # short ragged prompts, some nodes that see nothing, odd sizes
        _tree("tree_small_ragged", "small", 5, 13, 0, 517, "bf16", ragged=True, empty=True),
        # one online request with a large tree
        _tree("tree_single_60", "4b", 1, 60, 2048, 2048, "bf16", lse=True),
        # a serving batch over an 8-bit cache
        _tree("tree_batch_e4m3", "4b", 128, 16, 1024, 8192, "e4m3"),
        # large trees on a wide head: the most arithmetic
        _tree("tree_27b_64", "27b", 64, 64, 2048, 32768, "bf16"),
        # single-token decoding of long contexts: the most bytes
        _tree("decode_long_e4m3", "4b", 32, 1, 131072, 131072, "e4m3"),
    ]


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 1e14


def draw(rng):
    def logu(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    most = {op: max(_cost(c) for c in listed() if c["op"] == op) for op in ("rotary", "write", "read", "tree")}

    def rot(hd):
        dim = rng.choice([hd, hd, hd // 2, hd // 4, 2 * rng.randint(1, hd // 2)])
        kind = rng.choice(["none", "none", "linear", "ntk", "yarn"])
        if dim <= 2 and kind == "ntk":
            kind = "none"
        return _rot(dim, rng.choice(["half", "interleaved"]), kind, 1.0 if kind == "none" else rng.choice([2.0, 4.0, 8.0]),
                    rng.choice([4096, 32768]) if kind == "yarn" else 0, rng.choice([10000.0, 1e6]))

    op = rng.choice(["rotary", "write", "read", "tree", "tree", "tree"])
    head = rng.choice(list(HEADS))
    hd = HEADS[head][2]
    block = rng.choice([16, 16, 16, 32, 64])
    while True:
        if op == "rotary":
            c = _rotary(None, head, logu(1, 30000), logu(64, 1000000), rot(hd), rng.choice(["f32", "bf16", "bf16"]),
                        rng.random() < 0.4)
        elif op == "write":
            pick = rng.choice([0, 0, logu(2, 64)])
            hi = rng.randint(1, pick) if pick else logu(1, 8192)
            c = _cache(None, "write", head, logu(1, 200), max(1, hi // rng.choice([1, 2, 8])), hi, logu(1, 8192),
                       rng.choice(["bf16", "e4m3", "e4m3", "f32"]), rng.choice(["bf16", "f32"]),
                       rot(hd) if rng.random() < 0.5 else None, pick, block)
        elif op == "read":
            hi = logu(1, 8192)
            c = _cache(None, "read", head, logu(1, 200), max(1, hi // rng.choice([1, 2, 8])), hi, logu(1, 2000),
                       rng.choice(["bf16", "e4m3", "e4m3", "f32"]), rng.choice(["bf16", "f32"]), None, 0, block)
        else:
            hi = logu(16, 131072)
            lo = rng.choice([hi, hi // 2, hi // 8, 0])
            dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
            empty = rng.random() < 0.2
            c = _tree(None, head, logu(1, 128), rng.choice([1, 1, logu(2, 64), logu(2, 64), logu(65, 200)]), lo, hi,
                      "f32" if dtype == "f32" else rng.choice(["bf16", "e4m3"]), dtype, block, rng.random() < 0.4, empty,
                      not empty and rng.random() < 0.5)
        if _cost(c) <= 0.9 * most[op] and _room(c) <= 40e9:
            return c


def _room(c):
    """Bytes of the largest of the plain form's tensors."""
    nq, nkv, hd = HEADS[c["head"]]
    if c["op"] == "rotary":
        return c["rows"] * (nq + nkv) * hd * 8
    held = c["batch"] * (c["hi"] + c.get("start", 0)) * nkv * hd * 8
    return max(held, c["batch"] * c["hi"] * nq * c["nodes"] * 4) if c["op"] == "tree" else held


# ---------------------------------------------------------------- what belongs to the case

def _rng(c):
    return np.random.Generator(np.random.PCG64([c["batch"], c["lo"], c["hi"]]))


def _counts(c):
    """Rows (write, read) or cached tokens (tree) of each sequence: log-uniform in [lo, hi]."""
    if c["lo"] == c["hi"]:
        return np.full(c["batch"], c["lo"], dtype=np.int64)
    lo = max(c["lo"], 1)
    x = np.rint(np.exp(_rng(c).uniform(math.log(lo), math.log(c["hi"]), size=c["batch"]))).astype(np.int64)
    x = np.clip(x, lo, c["hi"])
    if c["lo"] == 0:
        x[0] = 0
    return x


def _starts(c):
    return _rng(c).integers(0, c["start"] + 1, size=c["batch"]) if c["start"] else np.zeros(c["batch"], dtype=np.int64)


def _nodes(c):
    n = np.full(c["batch"], c["nodes"], dtype=np.int64)
    if c["ragged"]:
        n = _rng(c).integers(0, c["nodes"] + 1, size=c["batch"])
        n[-1] = c["nodes"]
    return n


def _sees(c):
    """[B, T, T] bool: node i sees its ancestors and itself in a random tree (parents drawn
    among the nodes shortly before); with empty, every fifth node sees none."""
    rng, t = _rng(c), c["nodes"]
    see = np.zeros((c["batch"], t, t), dtype=bool)
    for i in range(t):
        see[:, i, i] = True
        if i:
            parent = np.maximum(0, i - 1 - rng.integers(0, 4, size=c["batch"]))
            see[:, i] |= see[np.arange(c["batch"]), parent]
    if c["empty"]:
        see[:, ::5] = False
    return see


# ---------------------------------------------------------------- inputs

def _frequencies(c):
    """Radians per position of the dim / 2 pairs, and the factor on the rotated values."""
    dim, f = c["rot_dim"], c["rot_factor"]
    p = np.arange(dim // 2, dtype=np.float64)
    base = c["rot_base"] * (f ** (dim / (dim - 2.0)) if c["rot_scaling"] == "ntk" else 1.0)
    theta = base ** (-2.0 * p / dim)
    if c["rot_scaling"] == "linear":
        theta = theta / f
    if c["rot_scaling"] == "yarn":  # turns within the trained length: at most 1 stretched, at least 32 kept
        g = np.clip((c["rot_original"] * theta / (2 * math.pi) - 1.0) / 31.0, 0.0, 1.0)
        theta = (1 - g) * theta / f + g * theta
        return theta, 0.1 * math.log(f) + 1.0
    return theta, 1.0


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, dtype, *shape, std=1.0):
    return torch.empty(shape, dtype=TYPES[dtype], device="cuda").normal_(0.0, std, generator=gen)


def _table(gen, need, block):
    """A block table of randomly placed blocks for `need` tokens of each sequence, and the pool's size."""
    per = torch.from_numpy(-(-need // block)).cuda()
    most, blocks = max(1, int(per.max())), int(per.sum()) + 4
    order = torch.randperm(blocks, generator=gen, device="cuda").to(torch.int32)
    col = torch.arange(most, device="cuda")
    at = torch.where(col < per[:, None], (torch.cumsum(per, 0) - per)[:, None] + col, torch.full_like(col, blocks - 1))
    return order[at].contiguous(), blocks


def _pool(gen, c, blocks, filled):
    """[blocks, KV heads, 2, block * head dim] and, in 8 bits, the exponents [.., 2, block]."""
    nq, nkv, hd = HEADS[c["head"]]
    shape, e = (blocks, nkv, 2, c["block"] * hd), None
    pool = torch.zeros(shape, dtype=torch.uint8 if c["cache"] == "e4m3" else TYPES[c["cache"]], device="cuda")
    if c["cache"] == "e4m3":
        e = torch.full((blocks, nkv, 2, c["block"]), 127, dtype=torch.uint8, device="cuda")
        pool = pool.view(TYPES["e4m3"])
    if filled:
        step = max(1, (1 << 29) // (nkv * 2 * c["block"] * hd))
        for b in range(0, blocks, step):
            part = pool[b:b + step]
            if e is None:
                part.normal_(0.0, 1.0, generator=gen)
            else:  # as quantised rows are: the largest of 128 normal values near 256, scales around 2^-7
                part.copy_(_normal(gen, "bf16", *part.shape, std=96.0).clamp_(-448.0, 448.0))
        if e is not None:
            e.random_(118, 122, generator=gen)
    return pool, e


def _words(see):
    """The mask's bits: word w of a node holds nodes 32 w .. 32 w + 31, lowest bit first."""
    b, t, _ = see.shape
    w = -(-t // 32)
    full = np.zeros((b, t, 32 * w), dtype=np.uint32)
    full[:, :, :t] = see
    words = (full.reshape(b, t, w, 32) << np.arange(32, dtype=np.uint32)).sum(-1, dtype=np.uint32)
    return torch.from_numpy(words.view(np.int32)).cuda()


def prepare(case, seed):
    c, gen = case, _gen(seed)
    nq, nkv, hd = HEADS[c["head"]]
    st = {"case": c}
    if c["op"] == "rotary":
        n = c["rows"]
        x = _normal(gen, c["dtype"], n, nq + 2 * nkv, hd)
        st.update(q=x[:, :nq], k=x[:, nq:nq + nkv],
                  positions=torch.randint(0, c["far"], (n,), generator=gen, device="cuda", dtype=torch.int32))
    elif c["op"] in ("write", "read"):
        rows, starts = _counts(c), _starts(c)
        n, first = int(rows.sum()), np.cumsum(rows) - rows
        table, blocks = _table(gen, starts + rows, c["block"])
        within = np.arange(n) - np.repeat(first, rows)
        st.update(seq_ids=torch.from_numpy(np.repeat(np.arange(c["batch"]), rows).astype(np.int32)).cuda(),
                  positions=torch.from_numpy((np.repeat(starts, rows) + within).astype(np.int32)).cuda(), src=None)
        pool, e = _pool(gen, c, blocks, c["op"] == "read")
        st.update(pool=pool, exponents=e, table=table, batch=c["batch"])
        if c["op"] == "write":
            if c["pick"]:  # the accepted path: rising nodes of each sequence's tree
                node = within * c["pick"] // np.repeat(np.maximum(rows, 1), rows)
                st["src"] = torch.from_numpy((np.repeat(np.arange(c["batch"]), rows) * c["pick"] + node).astype(np.int32)).cuda()
                n = c["batch"] * c["pick"]
            x = _normal(gen, c["dtype"], n, nq + 2 * nkv, hd)
            st.update(k=x[:, nq:nq + nkv], v=x[:, nq + nkv:])
    else:
        lens = _counts(c)
        table, blocks = _table(gen, lens, c["block"])
        pool, e = _pool(gen, c, blocks, True)
        x = _normal(gen, c["dtype"], c["batch"], c["nodes"], nq + 2 * nkv, hd)
        x[:, :, :nq] *= 1.5
        st.update(pool=pool, exponents=e, table=table, batch=c["batch"],
                  lens=torch.from_numpy(lens.astype(np.int32)).cuda(), longest=int(lens.max()),
                  q=x[:, :, :nq], k=x[:, :, nq:nq + nkv], v=x[:, :, nq + nkv:], mask=_words(_sees(c)),
                  counts=torch.from_numpy(_nodes(c).astype(np.int32)).cuda() if c["ragged"] else None,
                  out=torch.zeros((c["batch"], c["nodes"], nq, hd), dtype=TYPES[c["dtype"]], device="cuda"),
                  lse=torch.zeros((c["batch"], c["nodes"], nq), dtype=torch.float32, device="cuda") if c["lse"] else None)
    if own:  # the handles that a program keeps
        from paper_2608_28099_amd import ops
        if c.get("rot_dim"):
            st["rotary"] = ops.make_rotary(hd, rotary_dim=c["rot_dim"], base=c["rot_base"], layout=c["rot_layout"],
                                           scaling=c["rot_scaling"], factor=c["rot_factor"],
                                           original_positions=c["rot_original"])
        if "pool" in st:
            e = st["exponents"]
            st["store"] = ops.PagedCache(st["pool"][:, :, 0], st["pool"][:, :, 1], c["block"], st["table"],
                                         k_exponents=None if e is None else e[:, :, 0],
                                         v_exponents=None if e is None else e[:, :, 1])
    return st


# ---------------------------------------------------------------- one pass

def run(state):
    c = state["case"]
    if own:
        from paper_2608_28099_amd import ops
        if c["op"] == "rotary":
            return ops.rotary(state["rotary"], state["positions"], state["q"], state["k"], transpose=c["transpose"])
        if c["op"] == "tree":
            ops.tree_attention(state["store"], state["lens"], state["q"], state["k"], state["v"], mask=state["mask"],
                               counts=state["counts"], max_seq_len=state["longest"], out=state["out"], lse=state["lse"])
            return state["out"] if state["lse"] is None else (state["out"], state["lse"])
        if c["op"] == "write":
            ops.cache_write(state["store"], state["seq_ids"], state["positions"], state["k"], state["v"],
                            src_rows=state["src"], rotary=state.get("rotary"))
            if c["cache"] != "e4m3":
                return state["pool"]
        return ops.cache_read(state["store"], state["seq_ids"], state["positions"], TYPES[c["dtype"]])
    if c["op"] == "rotary":
        turn = _turns(c, state["positions"], c["transpose"])
        return _turned(c, state["q"], turn), _turned(c, state["k"], turn)
    if c["op"] == "tree":
        return _plain_tree(state)
    if c["op"] == "write":
        _plain_write(state)
        if c["cache"] != "e4m3":
            return state["pool"]
    return _plain_read(state)


def _turns(c, positions, transpose=False):
    """Angles in 64 bits, their cosines and sines rounded to 32."""
    theta, scale = _frequencies(c)
    a = positions.double()[:, None] * torch.from_numpy(theta).to(positions.device)
    cos, sin = (scale * torch.cos(a)).float()[:, None], (scale * torch.sin(a)).float()[:, None]
    return cos, -sin if transpose else sin


def _turned(c, x, turn):
    cos, sin = turn
    dim = c["rot_dim"]
    y = x.float()
    a, b = (y[..., :dim // 2], y[..., dim // 2:dim]) if c["rot_layout"] == "half" else (y[..., :dim:2], y[..., 1:dim:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    z = torch.cat([u, v], -1) if c["rot_layout"] == "half" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([z, y[..., dim:]], -1).to(x.dtype)


def _slots(state):
    c = state["case"]
    pos = state["positions"].long()
    return state["table"][state["seq_ids"].long(), pos // c["block"]].long(), pos % c["block"]


def _tiles(state):
    """Views of the pool: keys [blocks, KV heads, dims / x, block, x], values [blocks, KV heads, dims, block]."""
    pool, block = state["pool"], state["case"]["block"]
    pool = pool.view(torch.uint8) if pool.dtype == torch.float8_e4m3fn else pool
    x = 16 // pool.element_size()
    return pool[:, :, 0].unflatten(-1, (-1, block, x)), pool[:, :, 1].unflatten(-1, (-1, block))


def _quantised(x):
    """8-bit values and exponent bytes: the smallest power of two that brings a row within 448."""
    top = x.abs().amax(-1)
    part, power = torch.frexp(top)
    e = (power - torch.where(part <= 0.875, 9, 8)).clamp(-126, 127)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _plain_write(state):
    c = state["case"]
    k, v = state["k"], state["v"]
    if state["src"] is not None:
        k, v = k[state["src"].long()], v[state["src"].long()]
    k, v = k.float(), v.float()
    if c["rotated"]:
        k = _turned(c, k, _turns(c, state["positions"]))
    blk, slot = _slots(state)
    kt, vt = _tiles(state)
    if c["cache"] == "e4m3":
        k, ke = _quantised(k)
        v, ve = _quantised(v)
        state["exponents"][:, :, 0][blk, :, slot] = ke
        state["exponents"][:, :, 1][blk, :, slot] = ve
    kt[blk, :, :, slot, :] = k.unflatten(-1, (-1, kt.shape[-1])).to(kt.dtype)
    vt[blk, :, :, slot] = v.to(vt.dtype)


def _plain_read(state):
    c = state["case"]
    blk, slot = _slots(state)
    kt, vt = _tiles(state)
    k, v = kt[blk, :, :, slot, :].flatten(-2), vt[blk, :, :, slot]
    if c["cache"] == "e4m3":
        e = state["exponents"].float() - 127.0
        k = k.view(TYPES["e4m3"]).float() * torch.exp2(e[:, :, 0][blk, :, slot])[..., None]
        v = v.view(TYPES["e4m3"]).float() * torch.exp2(e[:, :, 1][blk, :, slot])[..., None]
    return k.to(TYPES[c["dtype"]]), v.to(TYPES[c["dtype"]])


def _plain_tree(state):
    c = state["case"]
    nq, nkv, hd = HEADS[c["head"]]
    batch, t, group = c["batch"], c["nodes"], nq // nkv
    table = state["table"].long()
    kt, vt = _tiles(state)
    k = kt[table].permute(0, 2, 1, 4, 3, 5).reshape(batch, nkv, -1, hd)   # [B, KV heads, tokens, dims]
    v = vt[table].permute(0, 2, 1, 4, 3).reshape(batch, nkv, -1, hd)
    if c["cache"] == "e4m3":
        e = torch.exp2(state["exponents"].float() - 127.0)
        k = k.view(TYPES["e4m3"]).float() * e[:, :, 0][table].transpose(1, 2).reshape(batch, nkv, -1)[..., None]
        v = v.view(TYPES["e4m3"]).float() * e[:, :, 1][table].transpose(1, 2).reshape(batch, nkv, -1)[..., None]
    k, v = k.float(), v.float()
    q = state["q"].float().unflatten(2, (nkv, group)).permute(0, 2, 1, 3, 4).reshape(batch, nkv, t * group, hd)
    q = q / math.sqrt(hd)
    kn, vn = state["k"].float().transpose(1, 2).contiguous(), state["v"].float().transpose(1, 2).contiguous()
    there = torch.arange(k.shape[2], device="cuda") < state["lens"][:, None]
    node = torch.arange(t, device="cuda")
    count = torch.full((batch,), t, device="cuda") if state["counts"] is None else state["counts"]
    see = (state["mask"][..., node // 32] >> (node % 32)) & 1
    see = (see > 0) & (node < count[:, None, None])
    see = see.repeat_interleave(group, 1)[:, None]                        # [B, 1, T group, T]
    sc = torch.matmul(q, k.transpose(2, 3)).masked_fill_(~there[:, None, None], -math.inf)
    sn = torch.matmul(q, kn.transpose(2, 3)).masked_fill_(~see, -math.inf)
    top = torch.maximum(sc.amax(-1, keepdim=True), sn.amax(-1, keepdim=True))
    top = torch.where(top == -math.inf, 0.0, top)
    sc, sn = sc.sub_(top).exp_(), sn.sub_(top).exp_()
    total = sc.sum(-1, keepdim=True) + sn.sum(-1, keepdim=True)
    v = v.masked_fill_(~there[:, None, :, None], 0.0)
    out = (torch.matmul(sc, v) + torch.matmul(sn, vn)) / torch.where(total == 0, 1.0, total)
    out = out.unflatten(2, (t, group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    live = (node < count[:, None])[..., None]
    state["out"].copy_(torch.where(live[..., None], out.to(state["out"].dtype), state["out"]))
    if state["lse"] is None:
        return state["out"]
    lse = (top + torch.log(total))[..., 0].unflatten(2, (t, group)).permute(0, 2, 1, 3).flatten(2, 3)
    state["lse"].copy_(torch.where(live, lse, state["lse"]))
    return state["out"], state["lse"]


# ---------------------------------------------------------------- work and the definition in 64 bits

def work(case):
    """Bytes: rows, ids and positions, and each stored token once (8-bit ones with their
    two exponents); operations: two per multiply-add of the products, three per rotated value."""
    c = case
    nq, nkv, hd = HEADS[c["head"]]
    esz = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "rotary":
        n = float(c["rows"])
        return {"bytes": n * ((nq + nkv) * hd * 2 * esz + 4), "flops": n * (nq + nkv) * c["rot_dim"] * 3}
    stored = nkv * 2 * (hd + 1 if c["cache"] == "e4m3" else hd * (2 if c["cache"] == "bf16" else 4))
    if c["op"] in ("write", "read"):
        n = float(_counts(c).sum())
        row = nkv * 2 * hd * esz
        rotate = 3.0 * n * nkv * c["rot_dim"]
        if c["op"] == "read":
            return {"bytes": n * (stored + row + 8), "flops": n * nkv * 2 * hd}
        back = stored + row if c["cache"] == "e4m3" else 0
        return {"bytes": n * (stored + row + back + (12 if c["pick"] else 8)), "flops": n * nkv * 4 * hd + rotate}
    lens, nodes = _counts(c).astype(np.float64), _nodes(c).astype(np.float64)
    byts = lens.sum() * (stored + 4 / c["block"]) + nodes.sum() * (2 * nq + 2 * nkv) * hd * esz
    byts += nodes.sum() * (4 * -(-c["nodes"] // 32) + (4 * nq if c["lse"] else 0))
    seen = c["batch"] * c["nodes"] * min(c["nodes"], 8)  # a node's ancestors, about
    return {"bytes": float(byts), "flops": 4.0 * hd * nq * float((lens * nodes).sum() + seen)}


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    nq, nkv, hd = HEADS[c["head"]]
    f64 = torch.float64

    def rotated(x, positions, backward=False):
        """Pairs as complex numbers, turned by e^(i a)."""
        theta, scale = _frequencies(c)
        dim, y = c["rot_dim"], x.to(f64).clone()
        ang = positions.to(f64)[:, None, None] * torch.from_numpy(theta).cuda()
        turn = torch.polar(torch.full_like(ang, scale), -ang if backward else ang)
        at = torch.arange(dim // 2, device="cuda")
        i0, i1 = (at, at + dim // 2) if c["rot_layout"] == "half" else (2 * at, 2 * at + 1)
        z = torch.complex(y[..., i0], y[..., i1]) * turn
        y[..., i0], y[..., i1] = z.real, z.imag
        return y

    if c["op"] == "rotary":
        return rotated(st["q"], st["positions"], c["transpose"]), rotated(st["k"], st["positions"], c["transpose"])

    block, table = c["block"], st["table"].long()
    x = 16 // st["pool"].element_size()
    dim = torch.arange(hd, device="cuda")

    def places(seqs, pos):
        """Flat indexes of one token's keys and values in a head's tile, and its block."""
        slot = (pos % block)[:, None]
        return table[seqs, pos // block], (dim // x * block + slot) * x + dim % x, dim * block + slot

    def fetch(pool, exps, blk, at, which, g):
        """[n, hd] of KV head g in 64 bits."""
        r = pool[:, g, which][blk[:, None], at].to(f64) if pool.dtype != TYPES["e4m3"] else \
            pool.view(torch.uint8)[:, g, which][blk[:, None], at].view(TYPES["e4m3"]).to(f64)
        if exps is None:
            return r
        slot = at[:, :1] // x % block if which == 0 else at[:, :1]
        return r * torch.exp2(exps[:, g, which][blk[:, None], slot].to(f64) - 127.0)

    if c["op"] in ("write", "read"):
        seqs, pos = st["seq_ids"].long(), st["positions"].long()
        blk, at_k, at_v = places(seqs, pos)
        if c["op"] == "read":
            return tuple(torch.stack([fetch(st["pool"], st["exponents"], blk, a, i, g) for g in range(nkv)], 1)
                         for i, a in enumerate((at_k, at_v)))
        k, v = st["k"].to(f64), st["v"].to(f64)
        if st["src"] is not None:
            k, v = k[st["src"].long()], v[st["src"].long()]
        if c["rotated"]:
            k = rotated(k, pos)
        if c["cache"] == "e4m3":
            def held(r):  # to the nearest of 8 steps per power of two, 2^-9 apart below 2^-6
                e = torch.ceil(torch.log2(r.abs().amax(-1, keepdim=True).clamp_min(1e-30) / 448.0))
                u = r / torch.exp2(e)
                step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3.0)
                return torch.round(u / step) * step * torch.exp2(e)
            return held(k), held(v)
        pool = st["pool"].to(f64)
        for g in range(nkv):
            pool[:, g, 0][blk[:, None], at_k] = k[:, g]
            pool[:, g, 1][blk[:, None], at_v] = v[:, g]
        return pool

    lens, nodes, see = _counts(c), _nodes(c), torch.from_numpy(_sees(c)).cuda()
    out = torch.zeros((c["batch"], c["nodes"], nq, hd), dtype=f64, device="cuda")
    lse = torch.zeros((c["batch"], c["nodes"], nq), dtype=f64, device="cuda")
    group = nq // nkv
    for b in range(c["batch"]):
        n, t = int(lens[b]), int(nodes[b])
        if t == 0:
            continue
        pos = torch.arange(n, device="cuda")
        blk, at_k, at_v = places(torch.full_like(pos, b), pos)
        for g in range(nkv):
            kk = torch.cat([fetch(st["pool"], st["exponents"], blk, at_k, 0, g), st["k"][b, :t, g].to(f64)])
            vv = torch.cat([fetch(st["pool"], st["exponents"], blk, at_v, 1, g), st["v"][b, :t, g].to(f64)])
            q = st["q"][b, :t, g * group:(g + 1) * group].to(f64).reshape(t * group, hd)
            ok = torch.cat([torch.ones((t, n), dtype=torch.bool, device="cuda"), see[b, :t, :t]], 1)
            s = (q @ kk.T) * hd ** -0.5
            s = s.masked_fill(~ok.repeat_interleave(group, 0), -math.inf)
            l = torch.logsumexp(s, -1)
            w = torch.exp(s - torch.where(l == -math.inf, 0.0, l)[:, None])
            out[b, :t, g * group:(g + 1) * group] = (w @ vv).reshape(t, group, hd)
            lse[b, :t, g * group:(g + 1) * group] = l.reshape(t, group)
    return (out, lse) if c["lse"] else out
