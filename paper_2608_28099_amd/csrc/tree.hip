// Attention of a tree of drafted tokens over the paged cache (include/sp_probe.h:
// sp_probe_tree_attention).
//
// Query rows of a KV head: row r = i * G + j is node i and the j-th of the G query
// heads that share it.  A wave takes 16 rows and the tokens of its sequence in units,
// first the cached ones, then the nodes, with one running softmax per row (maximum m in
// log2 units, sum l, output O not yet divided by l).
//
// Matrix-core operands (bf16 arithmetic).  S^T = K Q^T on 16x16x32 products: lane
// (li, la) = (lane % 16, lane / 16) holds of K the 8 dims 8 (la NC + c) .. + 7 of one
// token for product c, and receives the scores of query row li and four tokens.  Product h
// of a unit takes as its row m the token TPL (m / 4) + 4 h + m % 4, so that the lane's
// scores over all h are those of the TPL consecutive tokens TPL la .. : exactly its
// operand of O += P V, whose other operand is those tokens of dim 16 nt + li, side by side
// in the cache.  TPL is 8 (units of 32 tokens) for bf16 caches and nodes and 16 (units of
// 64) for 8-bit caches, so that either reads 16 bytes per lane at a time.  8-bit keys become
// bf16 with their exponent, exactly; the values' exponents go to the weights instead,
// exactly too (a power of two).
#include "common.h"
#include "ops.h"

namespace sp {
namespace {

__device__ __forceinline__ int64_t block_of(const StoreArg& st, int b, int t) {
  const int64_t at = (int64_t)b * st.mbps + (t >> st.bs_log2);
  const int64_t blk = st.block_table ? (int64_t)st.block_table[at] : at;
  return blk >= 0 && blk < st.num_blocks ? blk : 0;
}

__device__ __forceinline__ int count_of(const TreeParams& p, int b) {
  if (!p.counts) return p.nodes;
  const int n = p.counts[b];
  return n < 0 ? 0 : (n > p.nodes ? p.nodes : n);
}

// The nodes 32 u .. 32 u + 31 that node i of sequence b sees, of n.
__device__ __forceinline__ uint32_t seen_word(const TreeParams& p, int b, int i, int u, int n) {
  const int lim = p.mask ? n : min(n, i + 1);  // without a mask a chain
  const int left = lim - 32 * u;
  const uint32_t in = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0u;
  return p.mask ? p.mask[(int64_t)b * p.mask_stride + (int64_t)i * p.mask_words + u] & in : in;
}

// 8 values of a row, as two-byte words in order; `vec`: 16-byte aligned.
__device__ __forceinline__ u32x4 row8(const bf16* p, bool vec) {
  if (vec) return ld16v(p);
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = p[i];
  return __builtin_bit_cast(u32x4, w);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 E4M3 values (two words) to bf16, times a power of two.
__device__ __forceinline__ bf16x8 from_e4m3(uint32_t a, uint32_t b, float scale) {
  const bf16x2 w0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false);
  const bf16x2 w1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true);
  const bf16x2 w2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false);
  const bf16x2 w3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true);
  return bf16x8{w0[0], w0[1], w1[0], w1[1], w2[0], w2[1], w3[0], w3[1]};
}
__device__ __forceinline__ float exponent_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

template <int HD>
struct Rows {  // 16 query rows of a wave
  static constexpr int NC = HD / 32, NT = HD / 16;
  bf16x8 q[NC];   // Q[row li][8 (la NC + c) ..]
  f32x4 o[NT];    // O[row 4 la + r][16 nt + li]
  float m, l;     // row li: reference maximum (log2 units); the lane's part of the sum
};

// A row's reference maximum moves only when a score exceeds it by more than this (log2
// units), so weights stay below 2^8 between moves and most units skip the exchange
// across lanes and the rescaling of O.
constexpr float kRescaleLog2 = 8.0f;

// The lane's scores s (products not yet scaled; masked ones -inf) of NH * 4 tokens become
// weights 2^(s scale - m); where the maximum moves, l and o follow.
template <int HD, int NH>
__device__ __forceinline__ void softmax_step(Rows<HD>& st, f32x4 (&s)[NH], float scale, int la) {
  float mx = fmaxf(s[0][0], s[0][1]);
#pragma unroll
  for (int i = 2; i < 4 * NH; ++i) mx = fmaxf(mx, s[i / 4][i % 4]);
  mx *= scale;
  if (__any(mx > st.m + kRescaleLog2)) {
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    mx = fmaxf(mx, st.m);
    const float alpha = fast_exp2(st.m - mx);
    st.m = mx;
    st.l *= alpha;
    float ar[4];  // the factors of this lane's O rows 4 la + r
#pragma unroll
    for (int r = 0; r < 4; ++r) ar[r] = __shfl(alpha, 4 * la + r);
#pragma unroll
    for (int nt = 0; nt < Rows<HD>::NT; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) st.o[nt][r] *= ar[r];
  }
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[h][r] = fast_exp2(fmaf(s[h][r], scale, -st.m));
      st.l += s[h][r];
    }
}

// The weights of 8 tokens (scores h0 and h0 + 1) as a bf16 operand.  Rounded to nearest:
// each weight moves by at most 2^-8 of itself, what rounding the result to bf16 may cost too.
template <int NH>
__device__ __forceinline__ bf16x8 weights8(const f32x4 (&s)[NH], int h0) {
  bf16x8 w;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    w[r] = (bf16)s[h0][r];
    w[4 + r] = (bf16)s[h0 + 1][r];
  }
  return w;
}

// LDS image of a unit, in 16-byte pieces: NSUB runs of 16 tokens (each inside one
// block), their keys, then their values.  A run's keys: piece c * 16 + t = 16 bytes of dims
// of token t; its values: 8-bit: piece d = dim d of its 16 tokens; bf16: piece
// (2 nt + e) * 16 + i = dim 16 nt + i of its tokens 8 e .. 8 e + 7.  The 4-piece pad between
// the runs' keys lets the 16 lanes of a key fragment (4 or 8 tokens of every run) hit 16
// different 16-byte bank groups; a value fragment is 256 bytes in a row per 16 lanes.
// Pieces go from memory to LDS 64 at a time, each lane its own address.
template <int HD, bool E8>
struct Unit {
  static constexpr int NSUB = E8 ? 4 : 2, TOKENS = 16 * NSUB;
  static constexpr int SUB = E8 ? HD : 2 * HD;       // pieces of a run's keys, or of its values
  static constexpr int KP = SUB + 4, VB = NSUB * KP;
  static constexpr int EB = VB + NSUB * SUB;         // exponents: 64 words (keys 16, values 16, twice)
  static constexpr int PIECES = EB + (E8 ? 16 : 0);
  static constexpr int IPG = SUB / 64;               // loads of 64 pieces per run
  static constexpr int NI = 2 * NSUB * IPG;          // per unit
  static __device__ __forceinline__ int group_base(int gi) { return gi < NSUB ? gi * KP : VB + (gi - NSUB) * SUB; }
  // byte offset of piece q of a run from its first token's place in the block
  static __device__ __forceinline__ uint32_t key_off(int q, int bs) { return (uint32_t)((q >> 4) * bs + (q & 15)) * 16u; }
  static __device__ __forceinline__ uint32_t value_off(int q, int bs) {
    if (E8) return (uint32_t)(q * bs);
    return (uint32_t)((16 * (q >> 5) + (q & 15)) * bs * 2 + ((q >> 4) & 1) * 16);
  }
};

// Physical block ids of a split: two windows of kIdWin logical blocks, window w in half w & 1.
constexpr int kIdWin = 256;
constexpr int kStages = 3;

// Direct 4-byte loads into LDS: lane l's word lands at dst + 4 l (dst uniform).
__device__ __forceinline__ void ld4_to_lds(const void* addr, void* dst) {
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)dst;
  asm volatile("global_load_lds_dword %0, off" : : "v"(addr), "{m0}"(lds) : "memory");
}

// Wait until at most k units of PPL loads each remain in flight (k <= K).
template <int PPL, int K>
__device__ __forceinline__ void wait_units_le(int k) {
  if constexpr (K == 0) {
    wait_vmcnt<0>();
  } else {
    if (k >= K) wait_vmcnt<K * PPL>();
    else wait_units_le<PPL, K - 1>(k);
  }
}

// Bits of a word of E bytes per value whose first token is `keep` tokens before the end.
template <int E>
__device__ __forceinline__ uint32_t keep_mask(int keep) {
  return keep >= 4 / E ? ~0u : keep > 0 ? (1u << (8 * E * keep)) - 1 : 0u;
}

// One staged unit for the wave's ntw tiles: cached tokens, `limit` of them there, or (NODES,
// a bf16 unit) nodes, of which row li of tile t sees those in seen[t]; w keeps their weights.
template <int HD, bool E8, int TPW, bool NODES>
__device__ __forceinline__ void staged_unit(Rows<HD> (&st)[TPW], int ntw, const u32x4* sb, int limit,
                                            const uint32_t (&seen)[TPW], bf16x8 (&weights)[TPW], float scale, int li,
                                            int la) {
  using L = Unit<HD, E8>;
  constexpr int NC = HD / 32, NT = HD / 16, NH = E8 ? 4 : 2, TPL = 4 * NH;
  const int run = TPL * (li >> 2) / 16, first = TPL * (li >> 2) % 16 + (li & 3);  // of the lane's key
  f32x4 s[TPW][NH];
#pragma unroll
  for (int t = 0; t < TPW; ++t)
#pragma unroll
    for (int h = 0; h < NH; ++h) s[t][h] = f32x4{0.f, 0.f, 0.f, 0.f};
  if constexpr (E8) {
    const u32x4 ek = sb[L::EB + run];
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const float f = exponent_scale((ek[h] >> (8 * (li & 3))) & 0xffu);
#pragma unroll
      for (int q = 0; q < NC / 2; ++q) {
        const u32x4 w = sb[run * L::KP + (la * (NC / 2) + q) * 16 + first + 4 * h];
        const bf16x8 k0 = from_e4m3(w[0], w[1], f), k1 = from_e4m3(w[2], w[3], f);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
          if (t < ntw) {
            s[t][h] = mfma16x16x32_bf16(k0, st[t].q[2 * q], s[t][h]);
            s[t][h] = mfma16x16x32_bf16(k1, st[t].q[2 * q + 1], s[t][h]);
          }
      }
    }
  } else {
    u32x4 kf[NH][NC];
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int q = 0; q < NC; ++q) kf[h][q] = sb[run * L::KP + (la * NC + q) * 16 + first + 4 * h];
#pragma unroll
    for (int t = 0; t < TPW; ++t)
      if (t < ntw)
#pragma unroll
        for (int q = 0; q < NC; ++q)
#pragma unroll
          for (int h = 0; h < NH; ++h)
            s[t][h] = mfma16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[h][q]), st[t].q[q], s[t][h]);
  }
  // values are read once the scores' products are issued, into registers the keys held
  __builtin_amdgcn_sched_barrier(0);
  u32x4 vf[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
    vf[nt] = E8 ? sb[L::VB + la * L::SUB + 16 * nt + li]
                : sb[L::VB + (la >> 1) * L::SUB + (2 * nt + (la & 1)) * 16 + li];
  u32x4 ev = u32x4{0, 0, 0, 0};
  if constexpr (E8) ev = sb[L::EB + 4 + la];
  if constexpr (NODES) {
#pragma unroll
    for (int t = 0; t < TPW; ++t)
#pragma unroll
      for (int i = 0; i < TPL; ++i)
        if (!((seen[t] >> (TPL * la + i)) & 1)) s[t][i / 4][i % 4] = -INFINITY;
  } else if (limit < L::TOKENS) {  // a tail: tokens past the end may hold anything
    int lim = limit;
    asm volatile("" : "+s"(lim));  // (keeps the mask a branch that whole units skip)
#pragma unroll
    for (int t = 0; t < TPW; ++t)
#pragma unroll
      for (int i = 0; i < TPL; ++i)
        if (TPL * la + i >= lim) s[t][i / 4][i % 4] = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t keep = E8 ? keep_mask<1>(lim - (TPL * la + 4 * w)) : keep_mask<2>(lim - (TPL * la + 2 * w));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) vf[nt][w] &= keep;
      ev[w] &= keep;
    }
  }
#pragma unroll
  for (int t = 0; t < TPW; ++t)
    if (t < ntw) {
      softmax_step<HD, NH>(st[t], s[t], scale, la);
      if constexpr (E8)
#pragma unroll
        for (int i = 0; i < TPL; ++i) s[t][i / 4][i % 4] *= exponent_scale((ev[i / 4] >> (8 * (i % 4))) & 0xffu);
    }
  if constexpr (E8) {
    bf16x8 p0[TPW], p1[TPW];
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      p0[t] = weights8(s[t], 0);
      p1[t] = weights8(s[t], 2);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const bf16x8 v0 = from_e4m3(vf[nt][0], vf[nt][1], 1.f), v1 = from_e4m3(vf[nt][2], vf[nt][3], 1.f);
#pragma unroll
      for (int t = 0; t < TPW; ++t)
        if (t < ntw) {
          st[t].o[nt] = mfma16x16x32_bf16(p0[t], v0, st[t].o[nt]);
          st[t].o[nt] = mfma16x16x32_bf16(p1[t], v1, st[t].o[nt]);
        }
    }
  } else {
#pragma unroll
    for (int t = 0; t < TPW; ++t)
      if (t < ntw) {
        const bf16x8 p0 = weights8(s[t], 0);
        if constexpr (NODES) weights[t] = p0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          st[t].o[nt] = mfma16x16x32_bf16(p0, __builtin_bit_cast(bf16x8, vf[nt]), st[t].o[nt]);
      }
  }
}

// Nodes 32 u .. of n into the LDS image of a bf16 unit, by the whole workgroup.  Values that
// are not finite become 0 there (0 * NaN would carry a hidden node's values into every row);
// returns whether this lane met one.
template <int HD, int W>
__device__ __forceinline__ bool stage_nodes(const TreeParams& p, u32x4* sb, int b, int g, int u, int n, int tid) {
  using L = Unit<HD, false>;
  constexpr int C = HD / 8;
  const bf16* kb = (const bf16*)p.k.data + (int64_t)b * p.nodes * p.k.row + g * p.k.head;
  const bf16* vb = (const bf16*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
  bool odd = false;
  for (int i = tid; i < 16 * C; i += 64 * W) {
    const int c = i % C, t = 2 * (i / C), run = t >> 4;  // tokens t, t + 1; dims 8 c ..
    u32x4 v[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4 k = u32x4{0, 0, 0, 0};
      v[j] = k;
      const int node = 32 * u + t + j;
      if (node < n) {
        k = row8(kb + (int64_t)node * p.k.row + 8 * c, p.k_vec);
        v[j] = row8(vb + (int64_t)node * p.v.row + 8 * c, p.v_vec);
      }
      sb[run * L::KP + c * 16 + (t & 15) + j] = k;
#pragma unroll
      for (int w = 0; w < 4; ++w) {  // exponent bits all set: NaN or infinite
        const bool lo = (v[j][w] & 0x7f80u) == 0x7f80u, hi = (v[j][w] & 0x7f800000u) == 0x7f800000u;
        odd |= lo | hi;
        v[j][w] &= (lo ? 0xffff0000u : ~0u) & (hi ? 0xffffu : ~0u);
      }
    }
    const int e = (t >> 3) & 1;
#pragma unroll
    for (int d = 0; d < 8; ++d) {
      const int dim = 8 * c + d;
      const uint32_t a0 = (v[0][d / 2] >> (16 * (d & 1))) & 0xffffu, a1 = (v[1][d / 2] >> (16 * (d & 1))) & 0xffffu;
      uint32_t* piece = (uint32_t*)&sb[L::VB + run * L::SUB + (2 * (dim / 16) + e) * 16 + dim % 16];
      piece[(t & 7) / 2] = a0 | (a1 << 16);
    }
  }
  return odd;
}

// The values of nodes 32 u .. that are not finite, added to the rows that see them with weight w
// (row li's of nodes 8 la ..).
template <int HD>
__device__ __forceinline__ void add_odd_values(const TreeParams& p, Rows<HD>& st, bf16x8 weights, int b, int g, int u,
                                               int n, int li, int la) {
  const bf16* vb = (const bf16*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
  for (int t = 0; t < 32 && 32 * u + t < n; ++t) {
    float w = (float)weights[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) w = (t & 7) == e ? (float)weights[e] : w;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float wr = __shfl(w, 16 * (t >> 3) + 4 * la + r);
#pragma unroll
      for (int nt = 0; nt < HD / 16; ++nt) {
        const float x = to_f32(vb[(int64_t)(32 * u + t) * p.v.row + 16 * nt + li]);
        if (wr != 0.f && !(fabsf(x) <= 3.389531389e38f)) st.o[nt][r] = fmaf(wr, x, st.o[nt][r]);
      }
    }
  }
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// One workgroup per (group of query tiles, KV head; split; sequence): W waves, an even
// share of the group's tiles each (at most TPW).  The split's units pass through three LDS stages,
// loaded two units ahead; every fragment that a wave reads from LDS serves all its tiles.
// A sequence's last split takes the nodes too.  A sequence of one split is finished here,
// else its splits leave (m, l) and O for tree_merge.
template <int HD, bool E8, int W, int TPW>
__global__ __launch_bounds__(64 * W) void tree_split(const TreeParams p) {
  using L = Unit<HD, E8>;
  constexpr int NC = HD / 32, NT = HD / 16, NI = L::NI, NSUB = L::NSUB, U = L::TOKENS;
  constexpr int PPL = (NI + W - 1) / W, LOADS = PPL + (E8 ? 1 : 0), D = kStages - 1;
  static_assert(W <= 2 * NI && D * LOADS < 64, "loads in flight");
  __shared__ u32x4 stage[kStages][L::PIECES];
  __shared__ int blk_ids[2][kIdWin];
  __shared__ int odd_values[W];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, la = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < W);
  const int g = blockIdx.x % p.st.n_kv, qg = blockIdx.x / p.st.n_kv, b = blockIdx.z, s = blockIdx.y;
  const int n = count_of(p, b), rows = n * p.group;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
  const int t0 = s * p.split_len, t1 = min(len, t0 + p.split_len);
  if ((s > 0 && t0 >= len) || qg * p.n_tiles * 16 >= rows) return;
  const bool whole = len <= p.split_len, last = t1 == len;
  const int tb = wave * p.n_tiles / W, ntw = TPW == 1 ? 1 : (wave + 1) * p.n_tiles / W - tb;
  const int row0 = (qg * p.n_tiles + tb) * 16;

  Rows<HD> st[TPW];
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int row = min(row0 + 16 * t + li, rows - 1);
    const bf16* q = (const bf16*)p.q.data + ((int64_t)b * p.nodes + row / p.group) * p.q.row +
                    (int64_t)(g * p.group + row % p.group) * p.q.head;
#pragma unroll
    for (int c = 0; c < NC; ++c) st[t].q[c] = __builtin_bit_cast(bf16x8, row8(q + 8 * (la * NC + c), p.q_vec));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) st[t].o[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
    st[t].m = kNegBig;
    st[t].l = 0.f;
  }

  const StoreArg& c = p.st;
  constexpr int ESZ = E8 ? 1 : 2;
  const char* kbase = (const char*)c.k + g * c.k_sh * ESZ;
  const char* vbase = (const char*)c.v + g * c.v_sh * ESZ;
  const int bs = 1 << c.bs_log2, nunits = (t1 - t0 + U - 1) / U, lastu = nunits - 1;
  const int lb0 = t0 >> c.bs_log2, nlb = t1 > t0 ? ((t1 - 1) >> c.bs_log2) - lb0 + 1 : 0;
  const int* bt_row = c.block_table ? c.block_table + (int64_t)b * c.mbps + lb0 : nullptr;
  // The first two windows of block ids and the first nodes are under way together.
  constexpr int IDS = 2 * kIdWin / (64 * W) + (2 * kIdWin % (64 * W) != 0);
  int ids[IDS];
#pragma unroll
  for (int j = 0; j < IDS; ++j) {
    const int i = j * 64 * W + tid;
    ids[j] = bt_row && i < nlb ? bt_row[i] : 0;
  }
  if (last) {
    const bool odd = stage_nodes<HD, W>(p, stage[D], b, g, 0, n, tid);
    const bool any = __any(odd);
    if (lane == 0) odd_values[wave] = any;
  }
#pragma unroll
  for (int j = 0; j < IDS; ++j) {
    const int i = j * 64 * W + tid;
    if (i < 2 * kIdWin) blk_ids[i / kIdWin][i % kIdWin] = ids[j];
  }
  auto load_window = [&](int w) __attribute__((always_inline)) {
    for (int j = wave; j < kIdWin / 64; j += W)  // past the end: the last id again
      ld4_to_lds(bt_row + min(w * kIdWin + j * 64 + lane, nlb - 1), &blk_ids[w & 1][j * 64]);
  };
  uint32_t lane_off[PPL];
  int gsel[PPL], lds_piece[PPL];
#pragma unroll
  for (int j = 0; j < PPL; ++j) {
    const int slot = (j * W + wave) % NI;  // (a wave count that does not divide NI loads a few twice)
    gsel[j] = L::IPG % W == 0 ? j * W / L::IPG : slot / L::IPG;
    lds_piece[j] = L::group_base(gsel[j]) + (slot % L::IPG) * 64;
    const int q = (slot % L::IPG) * 64 + lane;
    lane_off[j] = gsel[j] < NSUB ? L::key_off(q, bs) : L::value_off(q, bs);
  }
  const int er = (lane >> 2) & 3;  // exponents: lanes 0..15 the keys', 16..31 the values', then both again
  // Loads are streaming (read once by this launch), unless another query group reads the
  // same blocks, or a unit takes less than its 64 bytes of a dim's row of values.
  const bool k_stream = p.n_qgroups == 1, v_stream = k_stream && bs * ESZ <= 64;
  auto issue = [&](int u, int buf) __attribute__((always_inline)) {
    int64_t blk[NSUB];
    int slot[NSUB];
#pragma unroll
    for (int r = 0; r < NSUB; ++r) {
      int t = t0 + U * u + 16 * r;
      t = t < t1 ? t : t0 + U * u;  // a run past the end reads the unit's first again
      const int rel = (t >> c.bs_log2) - lb0;
      slot[r] = t & (bs - 1);
      if (bt_row) blk[r] = __builtin_amdgcn_readfirstlane(blk_ids[((unsigned)rel / kIdWin) & 1][(unsigned)rel % kIdWin]);
      else blk[r] = (int64_t)b * c.mbps + lb0 + rel;
    }
    const char *kr[NSUB], *vr[NSUB];
#pragma unroll
    for (int r = 0; r < NSUB; ++r) {
      blk[r] = blk[r] >= 0 && blk[r] < c.num_blocks ? blk[r] : 0;
      kr[r] = kbase + blk[r] * c.k_sb * ESZ + slot[r] * 16;
      vr[r] = vbase + blk[r] * c.v_sb * ESZ + slot[r] * ESZ;
    }
#pragma unroll
    for (int j = 0; j < PPL; ++j) {
      const char* base = kr[0];
#pragma unroll
      for (int r = 1; r < NSUB; ++r) base = gsel[j] == r ? kr[r] : base;
#pragma unroll
      for (int r = 0; r < NSUB; ++r) base = gsel[j] == NSUB + r ? vr[r] : base;
      if (gsel[j] < NSUB ? k_stream : v_stream) ld16_to_lds(base, lane_off[j], &stage[buf][lds_piece[j]]);
      else ld16_to_lds<false>(base, lane_off[j], &stage[buf][lds_piece[j]]);
    }
    if constexpr (E8) {
      int64_t eb = blk[0];
      int es = slot[0];
#pragma unroll
      for (int r = 1; r < NSUB; ++r) {
        eb = er == r ? blk[r] : eb;
        es = er == r ? slot[r] : es;
      }
      const uint8_t* e = lane & 16 ? c.v_exp : c.k_exp;
      ld4_to_lds(e + eb * c.e_sb + g * c.e_sh + es + 4 * (lane & 3), &stage[buf][L::EB]);
    }
  };
  // entering window w when issuing unit v: window w + 1 replaces w - 1, which no later unit reads
  auto next_window = [&](int v) __attribute__((always_inline)) {
    const int w = (((t0 + U * v) >> c.bs_log2) - lb0) / kIdWin;
    const int wp = (((t0 + U * (v - 1)) >> c.bs_log2) - lb0) / kIdWin;
    if (bt_row && w != wp && (w + 1) * kIdWin < nlb) load_window(w + 1);
  };
  uint32_t seen[TPW];
  bf16x8 weights[TPW];
  // nothing that the compiler counts stays in flight past this point
  wait_vmcnt<0>();
  lds_barrier();
#pragma unroll
  for (int v = 0; v < D; ++v)
    if (v <= lastu) issue(v, v);
  if (last)  // the nodes, from the stage that unit D will take, while the first units arrive
    for (int u = 0; 32 * u < n; ++u) {
      if (u > 0) {
        lds_barrier();
        const bool odd = stage_nodes<HD, W>(p, stage[D], b, g, u, n, tid);
        const bool any = __any(odd);
        if (lane == 0) odd_values[wave] = any;
        lds_barrier();
      }
#pragma unroll
      for (int t = 0; t < TPW; ++t) seen[t] = seen_word(p, b, min(row0 + 16 * t + li, rows - 1) / p.group, u, n);
      staged_unit<HD, false, TPW, true>(st, ntw, stage[D], 32, seen, weights, p.scale_log2, li, la);
      bool odd = false;
#pragma unroll
      for (int w = 0; w < W; ++w) odd |= odd_values[w] != 0;
      if (odd)
#pragma unroll
        for (int t = 0; t < TPW; ++t)
          if (t < ntw) add_odd_values<HD>(p, st[t], weights[t], b, g, u, n, li, la);
    }
  int buf = 0;
  for (int u = 0; u < nunits; ++u) {
    // this wave's loads of unit u have landed; after the barrier everyone's have, and all are past unit u - 1
    wait_units_le<LOADS, D - 1>(min(u + D - 1, lastu) - u);
    lds_barrier();
    if (u + D <= lastu) {
      issue(u + D, buf == 0 ? kStages - 1 : buf - 1);
      next_window(u + D);
    }
    staged_unit<HD, E8, TPW, false>(st, ntw, stage[buf], t1 - (t0 + U * u), seen, weights, p.scale_log2, li, la);
    buf = buf == kStages - 1 ? 0 : buf + 1;
  }
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    const int r0 = row0 + 16 * t;
    if (t >= ntw || r0 >= rows) continue;
    float l = st[t].l;
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (whole) {
      const int row = r0 + li;
      if (p.lse && la == 0 && row < rows)
        p.lse[((int64_t)b * p.nodes + row / p.group) * (p.st.n_kv * p.group) + g * p.group + row % p.group] = lse_of(st[t].m, l);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float lr = __shfl(l, 4 * la + r);
        const float inv = lr == 0.f ? 0.f : 1.0f / lr;
        const int orow = r0 + 4 * la + r;
        if (orow >= rows) continue;
        bf16* o = (bf16*)p.out.data + ((int64_t)b * p.nodes + orow / p.group) * p.out.row +
                  (int64_t)(g * p.group + orow % p.group) * p.out.head;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) o[16 * nt + li] = (bf16)(st[t].o[nt][r] * inv);
      }
    } else {
      const int64_t prow = (((int64_t)b * p.st.n_kv + g) * p.max_splits + s) * p.r_alloc + r0;
      if (la == 0) p.ml_part[prow + li] = make_float2(st[t].m, l);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int r = 0; r < 4; ++r) p.o_part[(prow + 4 * la + r) * HD + 16 * nt + li] = st[t].o[nt][r];
    }
  }
}

// Joins the splits of the sequences that have several: one wave per query row, its lanes
// along the dims, every split's O weighted by 2^(m - the largest m).
template <int HD, typename T>
__global__ __launch_bounds__(256) void tree_merge(const TreeParams p) {
  constexpr int V = HD / 64;
  const int lane = threadIdx.x & 63, g = blockIdx.y, b = blockIdx.z;
  const int row = 4 * blockIdx.x + (threadIdx.x >> 6);
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
  if (len <= p.split_len || row >= count_of(p, b) * p.group) return;
  const int ns = (len + p.split_len - 1) / p.split_len;
  const int64_t base = ((int64_t)b * p.st.n_kv + g) * p.max_splits * p.r_alloc + row;
  float m = kNegBig;
  for (int s = lane; s < ns; s += 64) m = fmaxf(m, p.ml_part[base + (int64_t)s * p.r_alloc].x);
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  float l = 0.f, acc[V] = {};
#pragma unroll 4
  for (int s = 0; s < ns; ++s) {
    const int64_t at = base + (int64_t)s * p.r_alloc;
    const float2 ml = p.ml_part[at];
    const float w = fast_exp2(ml.x - m);
    l += w * ml.y;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float x = p.o_part[at * HD + V * lane + i];
      acc[i] += w * x;
    }
  }
  const int head = g * p.group + row % p.group;
  const int64_t node = (int64_t)b * p.nodes + row / p.group;
  if (p.lse && lane == 0) p.lse[node * (p.st.n_kv * p.group) + head] = lse_of(m, l);
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  T* o = (T*)p.out.data + node * p.out.row + (int64_t)head * p.out.head;
#pragma unroll
  for (int i = 0; i < V; ++i) o[V * lane + i] = from_f32<T>(acc[i] * inv);
}

// ---------------------------------------------------------------- fp32
// The same rows with fp32 products: S^T = K Q^T, lane (li, la) holding dims 16 j + 4 la + e
// of token and row li, then O^T += V^T P^T with the scores of row li that the lane already
// has (tokens 4 la + r), so the running softmax needs no exchange but its maximum's.  One
// workgroup of 8 waves per (query tile, KV head; split; sequence); the waves take every
// eighth step of 16 tokens, cached ones and then, in the last split, nodes, straight from
// memory, and join through LDS in their order.
constexpr int kF32Waves = 8;

template <int HD>
__global__ __launch_bounds__(64 * kF32Waves) void tree_split_f32(const TreeParams p) {
  constexpr int NJ = HD / 16, NW = kF32Waves;
  __shared__ f32x4 osh[NW][NJ][64];
  __shared__ float2 mlsh[NW][64];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, la = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % p.st.n_kv, row0 = 16 * (blockIdx.x / p.st.n_kv), b = blockIdx.z, s = blockIdx.y;
  const int n = count_of(p, b), rows = n * p.group;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
  const int begin = s * p.split_len, end = min(len, begin + p.split_len);
  if (row0 >= rows || (s > 0 && begin >= len)) return;
  const int row = min(row0 + li, rows - 1), node = row / p.group, head = g * p.group + row % p.group;
  const int64_t bs = (int64_t)1 << p.st.bs_log2;
  f32x4 q[NJ], o[NJ];
  const float* qr = (const float*)p.q.data + ((int64_t)b * p.nodes + node) * p.q.row + (int64_t)head * p.q.head;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
#pragma unroll
    for (int e = 0; e < 4; ++e) q[j][e] = qr[16 * j + 4 * la + e];
    o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  float m = kNegBig, l = 0.f;
  // scores and values (zero where masked and not finite) of 16 tokens
  auto step = [&](f32x4 (&k)[NJ], f32x4 (&v)[NJ], uint32_t seen) __attribute__((always_inline)) {
    f32x4 sc = f32x4{0.f, 0.f, 0.f, 0.f}, sc2 = sc;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        sc = mfma16x16x4_f32(k[j][e], q[j][e], sc);
        sc2 = mfma16x16x4_f32(k[j][e + 1], q[j][e + 1], sc2);
      }
    float mx = m;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[r] = (seen >> (4 * la + r)) & 1 ? (sc[r] + sc2[r]) * p.scale_log2 : -INFINITY;
      mx = fmaxf(mx, sc[r]);
    }
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float alpha = exp2f(m - mx);
    m = mx;
    l *= alpha;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      sc[r] = exp2f(sc[r] - mx);
      l += sc[r];
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) o[j] *= alpha;
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NJ; ++j) o[j] = mfma16x16x4_f32(v[j][r], sc[r], o[j]);
    return sc;
  };
  for (int t0 = begin + 16 * wave; t0 < end; t0 += 16 * NW) {
    const int limit = end - t0;
    const int64_t blk = block_of(p.st, b, t0), slot = t0 & (bs - 1);
    const float* kt = (const float*)p.st.k + blk * p.st.k_sb + g * p.st.k_sh + (la * bs + slot + li) * 4;
    const float* vt = (const float*)p.st.v + blk * p.st.v_sb + g * p.st.v_sh + li * bs + slot + 4 * la;
    f32x4 k[NJ], v[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      k[j] = *reinterpret_cast<const f32x4*>(kt + 16 * j * bs);
      v[j] = *reinterpret_cast<const f32x4*>(vt + 16 * j * bs);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[j][r] = 4 * la + r < limit ? v[j][r] : 0.f;
    }
    step(k, v, limit >= 16 ? 0xffffu : (1u << limit) - 1);
  }
  const float* kb = (const float*)p.k.data + (int64_t)b * p.nodes * p.k.row + g * p.k.head;
  const float* vb = (const float*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
  // node steps go on where the cached ones end
  const int ahead = (wave + NW - (end - begin + 15) / 16 % NW) % NW;
  for (int t0 = end == len ? 16 * ahead : n; t0 < n; t0 += 16 * NW) {
    const uint32_t seen = (seen_word(p, b, node, t0 >> 5, n) >> (t0 & 16)) & 0xffffu;
    const float* kr = kb + (int64_t)min(t0 + li, n - 1) * p.k.row;
    f32x4 k[NJ], v[NJ];
    bool odd = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        k[j][r] = kr[16 * j + 4 * la + r];
        const int t = t0 + 4 * la + r;
        v[j][r] = t < n ? vb[(int64_t)t * p.v.row + 16 * j + li] : 0.f;
        if (!(fabsf(v[j][r]) <= 3.402823466e38f)) {
          odd = true;
          v[j][r] = 0.f;
        }
      }
    const f32x4 sc = step(k, v, seen);
    if (__any(odd)) {
      // values that are not finite, taken out of the products above, reach only the rows that
      // see them: O^T has this lane's row li, dims 16 j + 4 la + r
      for (int t = 0; t < 16 && t0 + t < n; ++t) {
        float w = sc[0];
#pragma unroll
        for (int e = 1; e < 4; ++e) w = (t & 3) == e ? sc[e] : w;
        w = __shfl(w, 16 * (t >> 2) + li);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float x = vb[(int64_t)(t0 + t) * p.v.row + 16 * j + 4 * la + r];
            if (w != 0.f && !(fabsf(x) <= 3.402823466e38f)) o[j][r] = fmaf(w, x, o[j][r]);
          }
      }
    }
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  // join the waves; wave w finishes dims 16 w .. 16 w + 15 of the tile's rows
#pragma unroll
  for (int j = 0; j < NJ; ++j) osh[wave][j][lane] = o[j];
  mlsh[wave][lane] = make_float2(m, l);
  __syncthreads();
  if (wave >= NJ || row0 + li >= rows) return;
  float mg = mlsh[0][lane].x, lg = 0.f;
#pragma unroll
  for (int w = 1; w < NW; ++w) mg = fmaxf(mg, mlsh[w][lane].x);
  f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const float f = exp2f(mlsh[w][lane].x - mg);
    lg += mlsh[w][lane].y * f;
    x += osh[w][wave][lane] * f;
  }
  if (len <= p.split_len) {
    if (p.lse && wave == 0 && la == 0)
      p.lse[((int64_t)b * p.nodes + node) * (p.st.n_kv * p.group) + head] = lse_of(mg, lg);
    const float inv = lg == 0.f ? 0.f : 1.0f / lg;
    float* op = (float*)p.out.data + ((int64_t)b * p.nodes + node) * p.out.row + (int64_t)head * p.out.head + 16 * wave + 4 * la;
#pragma unroll
    for (int r = 0; r < 4; ++r) op[r] = x[r] * inv;
  } else {
    const int64_t prow = (((int64_t)b * p.st.n_kv + g) * p.max_splits + s) * p.r_alloc + row0 + li;
    if (wave == 0 && la == 0) p.ml_part[prow] = make_float2(mg, lg);
    *reinterpret_cast<f32x4*>(p.o_part + prow * HD + 16 * wave + 4 * la) = x;
  }
}

template <int HD, bool E8>
hipError_t split_typed(const TreeParams& p, dim3 grid, int waves, int tpw, hipStream_t s) {
#define SP_TREE_CASE(W_, TPW_)                                                            \
  if (waves == W_ && tpw == TPW_) {                                                       \
    hipLaunchKernelGGL((tree_split<HD, E8, W_, TPW_>), grid, dim3(64 * W_), 0, s, p);     \
    return hipGetLastError();                                                             \
  }
  SP_TREE_CASE(1, 1) SP_TREE_CASE(2, 1) SP_TREE_CASE(3, 1) SP_TREE_CASE(4, 1)
  SP_TREE_CASE(4, 2) SP_TREE_CASE(4, 3) SP_TREE_CASE(4, 4)
#undef SP_TREE_CASE
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_tree(const TreeParams& p, int storage, int hd, hipStream_t s) {
  const int rows = p.nodes * p.group;
  hipError_t e;
  if (storage == SP_F32) {
    if (p.split_len % 16 || (rows + 15) / 16 * 16 > p.r_alloc) return hipErrorInvalidValue;
    const dim3 grid(p.st.n_kv * ((rows + 15) / 16), p.max_splits, p.st.batch), block(64 * kF32Waves);
    if (hd == 128) hipLaunchKernelGGL((tree_split_f32<128>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_split_f32<64>), grid, block, 0, s, p);
    e = hipGetLastError();
  } else {
    const int tpw = (p.n_tiles + p.waves - 1) / p.waves;
    if (p.split_len % 64 || p.n_qgroups * p.n_tiles * 16 > p.r_alloc || (tpw == 1 && p.n_tiles != p.waves))
      return hipErrorInvalidValue;
    const dim3 grid(p.st.n_kv * p.n_qgroups, p.max_splits, p.st.batch);
    const bool e8 = storage == SP_E4M3;
    e = hd == 128 ? (e8 ? split_typed<128, true>(p, grid, p.waves, tpw, s) : split_typed<128, false>(p, grid, p.waves, tpw, s))
                  : (e8 ? split_typed<64, true>(p, grid, p.waves, tpw, s) : split_typed<64, false>(p, grid, p.waves, tpw, s));
  }
  if (e != hipSuccess || p.max_splits == 1) return e;
  const dim3 mgrid((rows + 3) / 4, p.st.n_kv, p.st.batch), block(256);
  if (storage == SP_F32) {
    if (hd == 128) hipLaunchKernelGGL((tree_merge<128, float>), mgrid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_merge<64, float>), mgrid, block, 0, s, p);
  } else {
    if (hd == 128) hipLaunchKernelGGL((tree_merge<128, bf16>), mgrid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_merge<64, bf16>), mgrid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace sp
