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
struct Rows {  // a wave's 16 query rows
  static constexpr int NC = HD / 32, NT = HD / 16;
  bf16x8 q[NC];   // Q[row li][8 (la NC + c) ..]
  f32x4 o[NT];    // O[row 4 la + r][16 nt + li]
  float m, l;     // row li: maximum (log2 units); the lane's part of the sum
};

// The scores s (log2 units, masked ones -inf) of the lane's NH * 4 tokens become weights;
// m, l and o move to the new maximum.
template <int HD, int NH>
__device__ __forceinline__ void softmax_step(Rows<HD>& st, f32x4 (&s)[NH], int la) {
  float mx = st.m;
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[h][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float alpha = fast_exp2(st.m - mx);
  st.m = mx;
  st.l *= alpha;
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[h][r] = fast_exp2(s[h][r] - mx);
      st.l += s[h][r];
    }
  float ar[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) ar[r] = __shfl(alpha, 4 * la + r);
#pragma unroll
  for (int nt = 0; nt < Rows<HD>::NT; ++nt)
#pragma unroll
    for (int r = 0; r < 4; ++r) st.o[nt][r] *= ar[r];
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

// One unit of cached tokens t0 .. (`limit` of them there are).
template <int HD, bool E8>
__device__ __forceinline__ void cache_unit(const TreeParams& p, Rows<HD>& st, int b, int g, int t0, int limit, int li,
                                           int la) {
  constexpr int NC = HD / 32, NT = HD / 16, NH = E8 ? 4 : 2, TPL = 4 * NH, X = E8 ? 16 : 8;
  const StoreArg& c = p.st;
  const int64_t bs = (int64_t)1 << c.bs_log2;
  // tokens past the end read the unit's first instead (they lie in a block the sequence owns)
  const int gk = TPL * (li >> 2), gv = TPL * la;  // first of the lane's group of tokens, as key and as value
  const int tk = t0 + (gk < limit ? gk : 0), tv = t0 + (gv < limit ? gv : 0);
  const int64_t bk = block_of(c, b, tk), bv = block_of(c, b, tv);
  const int64_t sk = tk & (bs - 1), sv = tv & (bs - 1);
  f32x4 s[NH];
#pragma unroll
  for (int h = 0; h < NH; ++h) s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
  u32x4 ev = u32x4{0, 0, 0, 0};
  if constexpr (E8) {
    const uint8_t* kb = (const uint8_t*)c.k + bk * c.k_sb + g * c.k_sh;
    const u32x4 ek = ld16v(c.k_exp + bk * c.e_sb + g * c.e_sh + sk);
    ev = ld16v(c.v_exp + bv * c.e_sb + g * c.e_sh + sv);
#pragma unroll
    for (int h = 0; h < NH; ++h) {
      const float scale = exponent_scale((ek[h] >> (8 * (li & 3))) & 0xffu);
#pragma unroll
      for (int q = 0; q < NC / 2; ++q) {
        const u32x4 w = ld16v(kb + ((int64_t)(la * (NC / 2) + q) * bs + sk + 4 * h + (li & 3)) * X);
        s[h] = mfma16x16x32_bf16(from_e4m3(w[0], w[1], scale), st.q[2 * q], s[h]);
        s[h] = mfma16x16x32_bf16(from_e4m3(w[2], w[3], scale), st.q[2 * q + 1], s[h]);
      }
    }
  } else {
    const bf16* kb = (const bf16*)c.k + bk * c.k_sb + g * c.k_sh;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int q = 0; q < NC; ++q) {
        const u32x4 w = ld16v(kb + ((int64_t)(la * NC + q) * bs + sk + 4 * h + (li & 3)) * X);
        s[h] = mfma16x16x32_bf16(__builtin_bit_cast(bf16x8, w), st.q[q], s[h]);
      }
  }
#pragma unroll
  for (int h = 0; h < NH; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) s[h][r] = TPL * la + 4 * h + r < limit ? s[h][r] * p.scale_log2 : -INFINITY;
  softmax_step<HD, NH>(st, s, la);
  if constexpr (E8) {
    // the values' exponents; slots past the end may hold anything
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        s[h][r] = TPL * la + 4 * h + r < limit ? s[h][r] * exponent_scale((ev[h] >> (8 * r)) & 0xffu) : 0.f;
    const bf16x8 p0 = weights8(s, 0), p1 = weights8(s, 2);
    const uint8_t* vb = (const uint8_t*)c.v + bv * c.v_sb + g * c.v_sh + sv;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      u32x4 w = ld16v(vb + (16 * nt + li) * bs);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int keep = limit - (TPL * la + 4 * h);  // the word's tokens that there are
        w[h] = keep >= 4 ? w[h] : keep > 0 ? w[h] & ((1u << (8 * keep)) - 1) : 0u;
      }
      st.o[nt] = mfma16x16x32_bf16(p0, from_e4m3(w[0], w[1], 1.f), st.o[nt]);
      st.o[nt] = mfma16x16x32_bf16(p1, from_e4m3(w[2], w[3], 1.f), st.o[nt]);
    }
  } else {
    const bf16x8 p0 = weights8(s, 0);
    const bf16* vb = (const bf16*)c.v + bv * c.v_sb + g * c.v_sh + sv;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      u32x4 w = ld16v(vb + (16 * nt + li) * bs);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int keep = limit - (TPL * la + 2 * h);
        w[h] = keep >= 2 ? w[h] : keep == 1 ? w[h] & 0xffffu : 0u;
      }
      st.o[nt] = mfma16x16x32_bf16(p0, __builtin_bit_cast(bf16x8, w), st.o[nt]);
    }
  }
}

// Nodes 32 u .. of n as keys and values.  `seen`: those that row li sees.
template <int HD>
__device__ __forceinline__ void node_unit(const TreeParams& p, Rows<HD>& st, int b, int g, int u, int n, uint32_t seen,
                                          int li, int la) {
  constexpr int NC = HD / 32, NT = HD / 16;
  const bf16* kb = (const bf16*)p.k.data + (int64_t)b * p.nodes * p.k.row + g * p.k.head;
  const bf16* vb = (const bf16*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
  f32x4 s[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    s[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16* kr = kb + (int64_t)min(32 * u + 8 * (li >> 2) + 4 * h + (li & 3), n - 1) * p.k.row;
#pragma unroll
    for (int q = 0; q < NC; ++q)
      s[h] = mfma16x16x32_bf16(__builtin_bit_cast(bf16x8, row8(kr + 8 * (la * NC + q), p.k_vec)), st.q[q], s[h]);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      s[h][r] = (seen >> (8 * la + 4 * h + r)) & 1 ? s[h][r] * p.scale_log2 : -INFINITY;
  }
  softmax_step<HD, 2>(st, s, la);
  const bf16x8 p0 = weights8(s, 0);
  bf16x8 v[NT];
  bool odd = false;  // a value that is not finite
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int t = 32 * u + 8 * la + e;
      v[nt][e] = t < n ? vb[(int64_t)t * p.v.row + 16 * nt + li] : (bf16)0.f;
      odd |= !(fabsf((float)v[nt][e]) <= 3.389531389e38f);
    }
  if (!__any(odd)) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) st.o[nt] = mfma16x16x32_bf16(p0, v[nt], st.o[nt]);
  } else {
    // 0 * NaN would carry a hidden node's values into every row: only what a row sees is added
    for (int t = 0; t < 32 && 32 * u + t < n; ++t) {
      float w = (float)p0[0];  // this lane's weight of row li for its token t % 8
#pragma unroll
      for (int e = 1; e < 8; ++e) w = (t & 7) == e ? (float)p0[e] : w;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float wr = __shfl(w, 16 * (t >> 3) + 4 * la + r);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float x = to_f32(vb[(int64_t)(32 * u + t) * p.v.row + 16 * nt + li]);
          st.o[nt][r] = wr != 0.f ? fmaf(wr, x, st.o[nt][r]) : st.o[nt][r];
        }
      }
    }
  }
}

// One wave per (16 query rows, KV head, sequence).
template <int HD, bool E8>
__global__ __launch_bounds__(64) void tree_wave(const TreeParams p) {
  constexpr int NC = HD / 32, NT = HD / 16, U = E8 ? 64 : 32;
  const int lane = threadIdx.x, li = lane & 15, la = lane >> 4;
  const int row0 = 16 * blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int n = count_of(p, b), rows = n * p.group;
  if (row0 >= rows) return;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
  const int row = min(row0 + li, rows - 1), node = row / p.group;
  Rows<HD> st;
  const bf16* q = (const bf16*)p.q.data + ((int64_t)b * p.nodes + node) * p.q.row +
                  (int64_t)(g * p.group + row % p.group) * p.q.head;
#pragma unroll
  for (int c = 0; c < NC; ++c) st.q[c] = __builtin_bit_cast(bf16x8, row8(q + 8 * (la * NC + c), p.q_vec));
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) st.o[nt] = f32x4{0.f, 0.f, 0.f, 0.f};
  st.m = kNegBig;
  st.l = 0.f;
  for (int t = 0; t < len; t += U) cache_unit<HD, E8>(p, st, b, g, t, len - t, li, la);
  for (int u = 0; 32 * u < n; ++u) node_unit<HD>(p, st, b, g, u, n, seen_word(p, b, node, u, n), li, la);
  float l = st.l;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
  if (p.lse && la == 0 && row0 + li < rows)
    p.lse[((int64_t)b * p.nodes + node) * (p.st.n_kv * p.group) + g * p.group + row % p.group] =
        l > 0.f || l != l ? (st.m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  float inv[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const float lr = __shfl(l, 4 * la + r);
    inv[r] = lr == 0.f ? 0.f : 1.0f / lr;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int orow = row0 + 4 * la + r;
    if (orow >= rows) continue;
    bf16* o = (bf16*)p.out.data + ((int64_t)b * p.nodes + orow / p.group) * p.out.row +
              (int64_t)(g * p.group + orow % p.group) * p.out.head;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[16 * nt + li] = (bf16)(st.o[nt][r] * inv[r]);
  }
}

// ---------------------------------------------------------------- fp32
// The same rows with fp32 products: S^T = K Q^T, lane (li, la) holding dims 16 j + 4 la + e
// of token and row li, then O^T += V^T P^T with the scores of row li that the lane already
// has (tokens 4 la + r), so the running softmax needs no exchange but its maximum's.
template <int HD>
__global__ __launch_bounds__(64) void tree_wave_f32(const TreeParams p) {
  constexpr int NJ = HD / 16;
  const int lane = threadIdx.x, li = lane & 15, la = lane >> 4;
  const int row0 = 16 * blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int n = count_of(p, b), rows = n * p.group;
  if (row0 >= rows) return;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
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
  for (int t0 = 0; t0 < len; t0 += 16) {
    const int limit = len - t0;
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
  for (int t0 = 0; t0 < n; t0 += 16) {
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
  if (row0 + li >= rows) return;
  if (p.lse && la == 0)
    p.lse[((int64_t)b * p.nodes + node) * (p.st.n_kv * p.group) + head] =
        l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  float* op = (float*)p.out.data + ((int64_t)b * p.nodes + node) * p.out.row + (int64_t)head * p.out.head;
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int r = 0; r < 4; ++r) op[16 * j + 4 * la + r] = o[j][r] * inv;
}

}  // namespace

hipError_t launch_tree(const TreeParams& p, int storage, int hd, int n_cus, hipStream_t s) {
  (void)n_cus;
  const dim3 grid((p.nodes * p.group + 15) / 16, p.st.n_kv, p.st.batch), block(64);
  if (storage == SP_F32) {
    if (hd == 128) hipLaunchKernelGGL((tree_wave_f32<128>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_wave_f32<64>), grid, block, 0, s, p);
  } else if (storage == SP_BF16) {
    if (hd == 128) hipLaunchKernelGGL((tree_wave<128, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_wave<64, false>), grid, block, 0, s, p);
  } else {
    if (hd == 128) hipLaunchKernelGGL((tree_wave<128, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_wave<64, true>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace sp
