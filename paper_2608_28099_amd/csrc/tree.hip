// Attention of a tree of drafted tokens over the paged cache (include/sp_probe.h:
// sp_probe_tree_attention).
//
// Query rows of a KV head: row r = i * G + j is node i and the j-th of the G query
// heads that share it.  A wave takes 16 or 32 rows and the tokens of its sequence's split in
// units, first the nodes, then the cached ones, with one running softmax per row (reference
// maximum m in log2 units, sum l, output O not yet divided by l).
//
// Matrix-core operands (bf16 arithmetic): S^T = K Q^T, then O^T += V^T P^T, so that the
// scores, the sum and the output of a row stay in the lanes of that row, and the scores that a
// lane receives of the first product are, as weights, its operand of the second.  For that the
// keys' tokens go to the rows of the first product in an order of their own (Wave16, Wave32).
// Units: 32 tokens of bf16 caches and nodes, 64 of 8-bit caches, 16 of fp32 (WaveF32), so that each reads 16 bytes
// per lane at a time.  8-bit keys meet the queries as they are, E4M3 with their exponents, in products of 128
// dims: a bf16 query is two E4M3 values (split_queries), so that two products replace the keys' conversion
// to bf16 (64 sequences of 6000 tokens, 320 rows: 794 -> 727 us).  8-bit values become bf16 bare, exactly; their exponents
// go to the weights, exactly too (a power of two).
#include <type_traits>

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

// 8 E4M3 values (two words) to bf16, times a power of two.
__device__ __forceinline__ bf16x8 from_e4m3(uint32_t a, uint32_t b, float scale) {
  return __builtin_bit_cast(
      bf16x8, u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, scale, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, scale, true))});
}
__device__ __forceinline__ float exponent_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte << 23);
}

__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// C + A B of E4M3 values: lane l has of row (column) l % 16 the 16 values of k from 16 (l / 16) and the 16 from 64 + 16 (l / 16).
// Powers of two 2^(e - 127): the lane's e scales the 32 values of k from 32 (l / 16).
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ f32x4 mfma16x16x128_e4m3(u32x8 a, u32x8 b, f32x4 c, int ea, int eb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_bit_cast(i32x8, a), __builtin_bit_cast(i32x8, b), c, 0, 0, 0, ea, 0, eb);
}

// Where they gain by it, waves raise their priority while they issue matrix products (s_setprio), so that of the
// waves of a SIMD, which run apart by what each waits for, one feeds the matrix cores while another takes its
// exponentials (64 sequences of 2K-32K tokens, 320 rows, bf16: 1200 us without, 1173 with; 48 of 1K-4K, 8-bit: 230, 224;
// waves of 16 rows with bf16 caches, no gain: 49.8, 50.6 for 16 sequences of 4000 tokens).

// A row's reference maximum moves only when a score exceeds it by more than this (log2
// units), so weights stay below 2^8 between moves and most units skip the exchange
// across lanes and the rescaling of O.
constexpr float kRescaleLog2 = 8.0f;

// The reference maximum of a row that has met no score yet: the lowest finite value, below which no finite score lies.
constexpr float kLowest = -3.402823466e38f;

// The weight's exponent s scale - m is one fma, exact but for its own rounding, while m is the product of the largest s rounded by
// itself: they differ by up to half a step of m, a power of two that all of the row's weights share and the division by their
// sum takes out.  Of maxima beyond kFineLog2 half a step is 1 and more, soon past the exponent's range, so there the difference
// is kept (RowState::rest) and taken off.  The test in every unit costs 1-2% (64 sequences of 2K-32K tokens, 320 rows, bf16:
// 1184 -> 1208 us; 64 of 6000, 320 rows, 8-bit: 712 -> 722).
constexpr float kFineLog2 = 16777216.0f;

// LDS image of a unit, in 16-byte pieces: NSUB runs of 16 tokens (each inside one
// block), their keys, then their values.  A run's keys: piece c * 16 + t = 16 bytes of dims
// of token t; its values: 8-bit: piece d = dim d of its 16 tokens; bf16: piece
// (2 nt + e) * 16 + i = dim 16 nt + i of its tokens 8 e .. 8 e + 7.  LDS serves a 16-byte read in groups
// of 16 lanes, 0-3, 12-15, 20-27 the first of them; the pad between the runs' keys (none for waves of 32
// rows) sends each group to 16 different 16-byte bank groups.  (Waves of 32 rows with a pad of 8 spent a third
// of their LDS cycles on conflicts.)  A value fragment is 256 bytes in a row per 16 lanes.
// Pieces go from memory to LDS 64 at a time, each lane its own address.
template <int HD, bool E8, int PAD>
struct Unit {
  static constexpr int NSUB = E8 ? 4 : 2, TOKENS = 16 * NSUB;
  static constexpr int SUB = E8 ? HD : 2 * HD;       // pieces of a run's keys, or of its values
  static constexpr int KP = SUB + PAD, VB = NSUB * KP;
  static constexpr int EB = VB + NSUB * SUB;         // exponents: per run 4 words the keys', 4 the values'
  static constexpr int PIECES = EB + (E8 ? 2 * NSUB : 0);
  static constexpr int PARTS = 1, IPG = SUB / 64;    // waves that share a run's keys, or its values; loads of 64 pieces each
  // byte offset of piece q of a run from its first token's place in the block
  static __device__ __forceinline__ uint32_t key_off(int q, int bs) { return (uint32_t)((q >> 4) * bs + (q & 15)) * 16u; }
  static __device__ __forceinline__ uint32_t value_off(int q, int bs) {
    if (E8) return (uint32_t)(q * bs);
    return (uint32_t)((16 * (q >> 5) + (q & 15)) * bs * 2 + ((q >> 4) & 1) * 16);
  }
};

// The image of a unit of fp32: one run of 16 tokens; keys: piece c * 16 + t = dims 4 c .. of token t; values: piece
// 4 d + e = dim d of tokens 4 e .. 4 e + 3.  Fragments are 1 KB in a row per wave.
template <int HD>
struct UnitF32 {
  static constexpr int NSUB = 1, TOKENS = 16, SUB = 4 * HD, KP = SUB, VB = SUB, EB = 2 * SUB, PIECES = 2 * SUB;
  static constexpr int PARTS = 2, IPG = SUB / 128;
  static __device__ __forceinline__ uint32_t key_off(int q, int bs) { return (uint32_t)((q >> 4) * bs + (q & 15)) * 16u; }
  static __device__ __forceinline__ uint32_t value_off(int q, int bs) { return (uint32_t)((q >> 2) * bs * 4 + (q & 3) * 16); }
};

// Physical block ids of a split: two windows of kIdWin logical blocks, window w in half w & 1.
constexpr int kIdWin = 256;

// Direct 4-byte loads into LDS: lane l's word lands at dst + 4 l (dst uniform).
__device__ __forceinline__ void ld4_to_lds(const void* addr, void* dst) {
  const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)dst;
  asm volatile("global_load_lds_dword %0, off" : : "v"(addr), "{m0}"(lds) : "memory");
}

// Bits of a word of E bytes per value whose first token is `keep` tokens before the end.
template <int E>
__device__ __forceinline__ uint32_t keep_mask(int keep) {
  return keep >= 4 / E ? ~0u : keep > 0 ? (1u << (8 * E * keep)) - 1 : 0u;
}

// Eight weights as a bf16 operand.  Rounded to nearest: each moves by at most 2^-8 of itself,
// what rounding the result to bf16 may cost too.  So the result is off by 0.0018-0.0023 of itself (root mean square) where weights in
// fp32 leave 0.0017, its own rounding.  What the rounding leaves as a second operand would give that back for one more
// product each: 64 sequences of 2K-32K tokens, 320 rows: 1184 -> 1520 us; 128 of 1K-8K 8-bit, 64 rows: 214 -> 276; single tokens of
// 32 sequences of 131072 8-bit: 1333 -> 1787, of 32768 bf16: 675 -> 679.
__device__ __forceinline__ bf16x8 weights8(const float* s) {
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = (bf16)s[i];
  return w;
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The running softmax of the row that a lane belongs to: O^T as NO vectors of OV values, the reference maximum m
// (log2 units) and the lane's part l of the sum.  Steps of S scores a lane.
template <int NO, typename OVec, int OV>
struct RowState {
  OVec o[NO];
  float m, l;
  float rest;  // largest score times scale - m, where that is taken off (else 0)
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int j = 0; j < NO; ++j)
#pragma unroll
      for (int r = 0; r < OV; ++r) o[j][r] = 0.f;
    m = kLowest;
    l = 0.f;
    rest = 0.f;
  }
  // Moves the reference maximum (and l and O) where one of the lane's scores s (products not yet scaled,
  // masked ones -inf) exceeds it by too much.  FROM: the first lane bit that tells lanes of a row apart.
  template <int S, int FROM>
  __device__ __forceinline__ void raise(const float (&s)[S], float scale) {
    float mx = fmaxf(s[0], s[1]);
#pragma unroll
    for (int i = 2; i < S; ++i) mx = fmaxf(mx, s[i]);
    if (__any(mx * scale > m + kRescaleLog2)) {
#pragma unroll
      for (int b = FROM; b < 64; b <<= 1) mx = fmaxf(mx, __shfl_xor(mx, b));
      const float top = mx * scale;
      if (top > m) rest = fabsf(top) > kFineLog2 ? fmaf(mx, scale, -top) : 0.f;
      mx = fmaxf(top, m);
      const float alpha = fast_exp2(m - mx);
      m = mx;
      l *= alpha;
#pragma unroll
      for (int j = 0; j < NO; ++j)
#pragma unroll
        for (int r = 0; r < OV; ++r) o[j][r] *= alpha;
    }
  }
  // Scores to weights 2^(s scale - m).
  template <int S>
  __device__ __forceinline__ void weigh(float (&s)[S], float scale) {
#pragma unroll
    for (int i = 0; i < S; ++i) s[i] = fmaf(s[i], scale, -m);
    if (__any(rest != 0.f))
#pragma unroll
      for (int i = 0; i < S; ++i) s[i] -= rest;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      s[i] = fast_exp2(s[i]);
      l += s[i];
    }
  }
};

// A wave of 16 rows on 16x16x32 products.  Lane (li, la) = (lane % 16, lane / 16) belongs to row li and
// holds of K the dims 8 (la NC + c) .. + 7 of one token for product c.  Product h of a unit takes as
// its row m the token TPL (m / 4) + 4 h + m % 4, so that the lane's scores over all h are those of the
// TPL consecutive tokens TPL la ..: its operand of the second product, whose other operand is those
// tokens of dim 16 nt + li, side by side in the cache (TPL 8 in bf16 units, 16 in 8-bit ones).
template <int HD, bool E8>
struct Wave16 {
  static constexpr int ROWS = 16, PAD = 4, NC = HD / 32, NT = HD / 16, NODES = 32;
  typedef bf16 T;
  typedef Unit<HD, E8, PAD> U;
  RowState<NT, f32x4, 4> st;  // o[nt][r]: dim 16 nt + 4 la + r
  bf16x8 q[NC];
  u32x8 qh, ql;       // 8-bit units: the lane's 32 dims of the row, q = qh 2^(eh - 127) + ql 2^(el - 127)
  int eh, el;
  int li, la;
  __device__ __forceinline__ Wave16(int lane) : li(lane & 15), la(lane >> 4) { st.clear(); }
  __device__ __forceinline__ int row() const { return li; }
  __device__ __forceinline__ void load_queries(const bf16* p, bool vec) {
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = __builtin_bit_cast(bf16x8, row8(p + 8 * (la * NC + c), vec));
  }

  // Queries for the products with 8-bit keys: dims 32 la .. + 31 of the row (head dim 64: 16 la .. + 15, of which the
  // second 16 bytes hold ql).  qh: E4M3 with the power of two that brings the row within 448; ql: what is left, times 16.
  // Eight significant bits of bf16 are four and four, so the two are exact down to scaled values of 2^-6.  Smaller ones may
  // be off by 2^-14, half of E4M3's least step over 16.  The row's largest becomes 224 to 448: that is below 2^-6 / 224 of it, by
  // 2^-14 / 224 of it at most (of rows within 448 2^-122, where the power ends: below 2^-128, by 2^-136).
  __device__ __forceinline__ void split_queries() {
    u32x4 w[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) w[c] = __builtin_bit_cast(u32x4, q[c]);
    uint32_t top = 0;  // the largest finite magnitude's bf16 bits
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t lo = w[c][i] & 0x7fffu, hi = (w[c][i] >> 16) & 0x7fffu;
        top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
    // 2^e with top <= 448 2^e = 1.75 2^(8 + e); e - 4 is kept within the scales' range
    int e = (int)(top >> 7) - 135 + ((top & 0x7fu) > 0x60u ? 1 : 0);
    e = e < -122 ? -122 : e;
    const float f = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        int h = 0, l = 0;
        float x[4], r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = w[c][i + j / 2];
          x[j] = __builtin_bit_cast(float, j & 1 ? v & 0xffff0000u : v << 16) * f;
          x[j] = is_finite(x[j]) ? x[j] : __builtin_nanf("");
        }
        h = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], h, false);
        h = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], h, true);
        r[0] = 16.f * (x[0] - __builtin_amdgcn_cvt_f32_fp8(h, 0));
        r[1] = 16.f * (x[1] - __builtin_amdgcn_cvt_f32_fp8(h, 1));
        r[2] = 16.f * (x[2] - __builtin_amdgcn_cvt_f32_fp8(h, 2));
        r[3] = 16.f * (x[3] - __builtin_amdgcn_cvt_f32_fp8(h, 3));
        l = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], l, false);
        l = __builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], l, true);
        qh[2 * c + i / 2] = (uint32_t)h;
        ql[2 * c + i / 2] = (uint32_t)l;
      }
    eh = e + 127;
    el = e + 123;
    if (HD == 64) {
#pragma unroll
      for (int i = 0; i < 4; ++i) qh[4 + i] = ql[i];
      eh = la < 2 ? eh : el;
    }
  }

  template <bool U8>
  __device__ __forceinline__ void scores(float (&s)[U8 ? 16 : 8], const u32x4* sb) const {
    using L = Unit<HD, U8, PAD>;
    constexpr int NH = U8 ? 4 : 2, TPL = 4 * NH;
    const int run = TPL * (li >> 2) / 16, first = TPL * (li >> 2) % 16 + (li & 3);  // of the lane's key
    f32x4 d[NH];
#pragma unroll
    for (int h = 0; h < NH; ++h) d[h] = f32x4{0.f, 0.f, 0.f, 0.f};
    if constexpr (U8) {
      const u32x4 ek = sb[L::EB + 2 * run];
      constexpr int PL = HD / 64;  // pieces of a lane
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const u32x4* at = &sb[run * L::KP + la * PL * 16 + first + 4 * h];
        const u32x8 k = __builtin_shufflevector(at[0], at[16 * (PL - 1)], 0, 1, 2, 3, 4, 5, 6, 7);
        const int e = (int)((ek[h] >> (8 * (li & 3))) & 0xffu);
        d[h] = mfma16x16x128_e4m3(k, qh, d[h], e, eh);
        if (HD == 128) d[h] = mfma16x16x128_e4m3(k, ql, d[h], e, el);
      }
    } else {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int h = 0; h < NH; ++h)
          d[h] = mfma16x16x32_bf16(__builtin_bit_cast(bf16x8, sb[run * L::KP + (la * NC + c) * 16 + first + 4 * h]), q[c], d[h]);
    }
#pragma unroll
    for (int i = 0; i < TPL; ++i) s[i] = d[i / 4][i % 4];
  }

  // Scores, weights and values of a staged unit of cached tokens; in a tail `limit` tokens of it exist, the
  // rest may hold anything.
  __device__ __forceinline__ void cached_unit(const u32x4* sb, bool tail, int limit, float scale) {
    using L = Unit<HD, E8, PAD>;
    constexpr int TPL = E8 ? 16 : 8;
    float s[TPL];
    if (E8) __builtin_amdgcn_s_setprio(1);
    scores<E8>(s, sb);
    if (E8) __builtin_amdgcn_s_setprio(0);
    // values are read once the scores' products are issued, into registers the keys held
    __builtin_amdgcn_sched_barrier(0);
    u32x4 v[NT], e = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      v[nt] = E8 ? sb[L::VB + la * L::SUB + 16 * nt + li] : sb[L::VB + (la >> 1) * L::SUB + (2 * nt + (la & 1)) * 16 + li];
    if constexpr (E8) e = sb[L::EB + 2 * la + 1];
    if (tail) {
      int lim = limit;
      asm volatile("" : "+s"(lim));  // (keeps the masks a branch that whole units skip)
#pragma unroll
      for (int i = 0; i < TPL; ++i)
        if (TPL * la + i >= lim) s[i] = -INFINITY;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t keep = E8 ? keep_mask<1>(lim - (16 * la + 4 * w)) : keep_mask<2>(lim - (8 * la + 2 * w));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) v[nt][w] &= keep;
        e[w] &= keep;
      }
    }
    st.template raise<TPL, 16>(s, scale);
    st.weigh(s, scale);
    if constexpr (E8) {
#pragma unroll
      for (int i = 0; i < TPL; ++i) s[i] *= exponent_scale((e[i / 4] >> (8 * (i % 4))) & 0xffu);
      const bf16x8 p0 = weights8(s), p1 = weights8(s + 8);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        st.o[nt] = mfma16x16x32_bf16(from_e4m3(v[nt][0], v[nt][1], 1.f), p0, st.o[nt]);
        st.o[nt] = mfma16x16x32_bf16(from_e4m3(v[nt][2], v[nt][3], 1.f), p1, st.o[nt]);
      }
    } else {
      const bf16x8 p0 = weights8(s);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) st.o[nt] = mfma16x16x32_bf16(__builtin_bit_cast(bf16x8, v[nt]), p0, st.o[nt]);
    }
    if (E8) __builtin_amdgcn_s_setprio(0);
  }

  // A staged unit of nodes, of which the lane's row sees those in `seen`.  odd(t, weight): called for every
  // node t that may hold values that are not finite, with the row's weight for it, if any_odd.
  template <typename F>
  __device__ __forceinline__ void node_unit(const u32x4* sb, uint32_t seen, float scale, bool any_odd, F odd) {
    using L = Unit<HD, false, PAD>;
    float s[8];
    scores<false>(s, sb);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!((seen >> (8 * la + i)) & 1)) s[i] = -INFINITY;
    st.template raise<8, 16>(s, scale);
    st.weigh(s, scale);
    const bf16x8 p0 = weights8(s);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      st.o[nt] = mfma16x16x32_bf16(
          __builtin_bit_cast(bf16x8, sb[L::VB + (la >> 1) * L::SUB + (2 * nt + (la & 1)) * 16 + li]), p0, st.o[nt]);
    if (any_odd)
      for (int t = 0; t < 32; ++t) {
        float w = (float)p0[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) w = (t & 7) == i ? (float)p0[i] : w;
        odd(t, __shfl(w, 16 * (t >> 3) + li));
      }
  }

  __device__ __forceinline__ float sum() const {
    float l = st.l;
    l += __shfl_xor(l, 16);
    return l + __shfl_xor(l, 32);
  }
  // f(first dim of four, the four values)
  template <typename F>
  __device__ __forceinline__ void each4(F f) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) f(16 * nt + 4 * la, st.o[nt]);
  }
  template <typename F>
  __device__ __forceinline__ void add4(F f) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int r = 0; r < 4; ++r) st.o[nt][r] = f(16 * nt + 4 * la + r, st.o[nt][r]);
  }
};

// A wave of 32 rows on 32x32x16 products, of bf16 caches: each fragment that it reads from LDS serves twice the
// rows.  Lane (lj, lh) = (lane % 32, lane / 32) belongs to row lj.  Row m of the first product is token
// 16 (m / 16) + 8 (m / 4 % 2) + 4 (m / 8 % 2) + m % 4 of the unit, so that score i of the lane is token
// 16 (i / 8) + 8 lh + i % 8: eight tokens of each run.
template <int HD, bool E8>
struct Wave32 {
  static constexpr int ROWS = 32, PAD = 0, NC = HD / 16, ND = HD / 32, NODES = 32;
  static_assert(!E8, "bf16 units");
  typedef bf16 T;
  typedef Unit<HD, E8, PAD> U;
  RowState<ND, f32x16, 16> st;  // o[dt][4 k + r]: dim 32 dt + 8 k + 4 lh + r
  bf16x8 q[NC];
  int lj, lh;
  __device__ __forceinline__ Wave32(int lane) : lj(lane & 31), lh(lane >> 5) { st.clear(); }
  __device__ __forceinline__ int row() const { return lj; }
  // product c takes dims 8 (2 c + lh) ..
  __device__ __forceinline__ void load_queries(const bf16* p, bool vec) {
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = __builtin_bit_cast(bf16x8, row8(p + 8 * (2 * c + lh), vec));
  }
  static __device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }

  __device__ __forceinline__ void bf16_scores(float (&s)[16], const u32x4* sb) const {
    using L = Unit<HD, false, PAD>;
    const int at = (lj >> 4) * L::KP + 8 * ((lj >> 2) & 1) + 4 * ((lj >> 3) & 1) + (lj & 3);
    f32x16 d;
#pragma unroll
    for (int i = 0; i < 16; ++i) d[i] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (c == NC / 2) __builtin_amdgcn_sched_barrier(0);  // (all keys at once take too many registers)
      d = mfma(__builtin_bit_cast(bf16x8, sb[at + (2 * c + lh) * 16]), q[c], d);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = d[i];
  }
  // the value fragment of dim tile dt and eight of the tokens of run t
  __device__ __forceinline__ u32x4 bf16_values(const u32x4* sb, int dt, int t) const {
    using L = Unit<HD, false, PAD>;
    return sb[L::VB + t * L::SUB + (2 * (2 * dt + (lj >> 4)) + lh) * 16 + (lj & 15)];
  }

  // keeps the first `keep` of the fragments' eight tokens
  static __device__ __forceinline__ void clear_tail(u32x4 (&v)[ND], int keep) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const uint32_t bits = keep_mask<2>(keep - 2 * w);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) v[dt][w] &= bits;
    }
  }

  __device__ __forceinline__ void cached_unit(const u32x4* sb, bool tail, int limit, float scale) {
    float s[16];
    __builtin_amdgcn_s_setprio(1);
    bf16_scores(s, sb);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    u32x4 v[ND];
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) v[dt] = bf16_values(sb, dt, 0);
    if (tail) {
      int lim = limit;
      asm volatile("" : "+s"(lim));  // (keeps the masks a branch that whole units skip)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (16 * (i / 8) + 8 * lh + i % 8 >= lim) s[i] = -INFINITY;
      clear_tail(v, lim - 8 * lh);
    }
    st.template raise<16, 32>(s, scale);
    st.weigh(s, scale);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16x8 p = weights8(s + 8 * t);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) st.o[dt] = mfma(__builtin_bit_cast(bf16x8, v[dt]), p, st.o[dt]);
      if (t) break;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) v[dt] = bf16_values(sb, dt, 1);
      if (tail) clear_tail(v, limit - 16 - 8 * lh);
    }
    __builtin_amdgcn_s_setprio(0);
  }

  template <typename F>
  __device__ __forceinline__ void node_unit(const u32x4* sb, uint32_t seen, float scale, bool any_odd, F odd) {
    float s[16];
    bf16_scores(s, sb);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (!((seen >> (16 * (i / 8) + 8 * lh + i % 8)) & 1)) s[i] = -INFINITY;
    st.template raise<16, 32>(s, scale);
    st.weigh(s, scale);
    const bf16x8 p[2] = {weights8(s), weights8(s + 8)};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) st.o[dt] = mfma(__builtin_bit_cast(bf16x8, bf16_values(sb, dt, t)), p[t], st.o[dt]);
    if (any_odd)
      for (int t = 0; t < 32; ++t) {
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) w = (t & 7) + 8 * (t >> 4) == i ? (float)p[i / 8][i % 8] : w;
        odd(t, __shfl(w, 32 * ((t >> 3) & 1) + lj));
      }
  }

  __device__ __forceinline__ float sum() const { return st.l + __shfl_xor(st.l, 32); }
  template <typename F>
  __device__ __forceinline__ void each4(F f) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        f(32 * dt + 8 * k + 4 * lh, f32x4{st.o[dt][4 * k], st.o[dt][4 * k + 1], st.o[dt][4 * k + 2], st.o[dt][4 * k + 3]});
  }
  template <typename F>
  __device__ __forceinline__ void add4(F f) {
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
      for (int i = 0; i < 16; ++i) st.o[dt][i] = f(32 * dt + 8 * (i / 4) + 4 * lh + i % 4, st.o[dt][i]);
  }
};

// A wave of 16 rows with fp32 products (16x16x4): product (j, e) takes dims 16 j + 4 la + e of token and row li, and
// leaves the lane the scores of tokens 4 la + r of row li, its operands of the second.
template <int HD, bool>
struct WaveF32 {
  static constexpr int ROWS = 16, PAD = 0, NJ = HD / 16, NODES = 16;
  typedef float T;
  typedef UnitF32<HD> U;
  RowState<NJ, f32x4, 4> st;  // o[j][r]: dim 16 j + 4 la + r
  f32x4 q[NJ];
  int li, la;
  __device__ __forceinline__ WaveF32(int lane) : li(lane & 15), la(lane >> 4) { st.clear(); }
  __device__ __forceinline__ int row() const { return li; }
  __device__ __forceinline__ void load_queries(const float* p, bool vec) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const float* x = p + 16 * j + 4 * la;
      if (vec) q[j] = *reinterpret_cast<const f32x4*>(x);
      else q[j] = f32x4{x[0], x[1], x[2], x[3]};
    }
  }
  __device__ __forceinline__ void scores(float (&s)[4], const u32x4* sb) const {
    f32x4 d0 = f32x4{0.f, 0.f, 0.f, 0.f}, d1 = d0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const f32x4 k = __builtin_bit_cast(f32x4, sb[(4 * j + la) * 16 + li]);
      d0 = mfma16x16x4_f32(k[0], q[j][0], d0);
      d1 = mfma16x16x4_f32(k[1], q[j][1], d1);
      d0 = mfma16x16x4_f32(k[2], q[j][2], d0);
      d1 = mfma16x16x4_f32(k[3], q[j][3], d1);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) s[r] = d0[r] + d1[r];
  }
  __device__ __forceinline__ void products(const float (&s)[4], const f32x4 (&v)[NJ]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < NJ; ++j) st.o[j] = mfma16x16x4_f32(v[j][r], s[r], st.o[j]);
  }
  __device__ __forceinline__ void load_values(f32x4 (&v)[NJ], const u32x4* sb) const {
#pragma unroll
    for (int j = 0; j < NJ; ++j) v[j] = __builtin_bit_cast(f32x4, sb[U::VB + (16 * j + li) * 4 + la]);
  }
  __device__ __forceinline__ void cached_unit(const u32x4* sb, bool tail, int limit, float scale) {
    float s[4];
    scores(s, sb);
    __builtin_amdgcn_sched_barrier(0);
    f32x4 v[NJ];
    load_values(v, sb);
    if (tail)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (4 * la + r >= limit) {
          s[r] = -INFINITY;
#pragma unroll
          for (int j = 0; j < NJ; ++j) v[j][r] = 0.f;
        }
    st.template raise<4, 16>(s, scale);
    st.weigh(s, scale);
    products(s, v);
  }
  template <typename F>
  __device__ __forceinline__ void node_unit(const u32x4* sb, uint32_t seen, float scale, bool any_odd, F odd) {
    float s[4];
    scores(s, sb);
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (!((seen >> (4 * la + r)) & 1)) s[r] = -INFINITY;
    st.template raise<4, 16>(s, scale);
    st.weigh(s, scale);
    f32x4 v[NJ];
    load_values(v, sb);
    products(s, v);
    if (any_odd)
      for (int t = 0; t < 16; ++t) {
        float w = s[0];
#pragma unroll
        for (int r = 1; r < 4; ++r) w = (t & 3) == r ? s[r] : w;
        odd(t, __shfl(w, 16 * (t >> 2) + li));
      }
  }
  __device__ __forceinline__ float sum() const {
    float l = st.l;
    l += __shfl_xor(l, 16);
    return l + __shfl_xor(l, 32);
  }
  template <typename F>
  __device__ __forceinline__ void each4(F f) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) f(16 * j + 4 * la, st.o[j]);
  }
  template <typename F>
  __device__ __forceinline__ void add4(F f) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) st.o[j][r] = f(16 * j + 4 * la + r, st.o[j][r]);
  }
};

// Nodes 32 u .. of n into the LDS image of a bf16 unit, by the whole workgroup.  Values that
// are not finite become 0 there (0 * NaN would carry a hidden node's values into every row);
// returns whether this lane met one.
template <int HD, int W, int PAD>
__device__ __forceinline__ bool stage_nodes(const TreeParams& p, u32x4* sb, int b, int g, int u, int n, int tid) {
  using L = Unit<HD, false, PAD>;
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

// The same for nodes 16 u .. and a unit of fp32.
template <int HD, int W>
__device__ __forceinline__ bool stage_nodes_f32(const TreeParams& p, u32x4* sb, int b, int g, int u, int n, int tid) {
  using L = UnitF32<HD>;
  const float* kb = (const float*)p.k.data + (int64_t)b * p.nodes * p.k.row + g * p.k.head;
  const float* vb = (const float*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
  bool odd = false;
  for (int i = tid; i < 4 * HD; i += 64 * W) {
    const int c = i % (HD / 4), t = i / (HD / 4), node = 16 * u + t;  // dims 4 c .. of node t
    f32x4 k = f32x4{0.f, 0.f, 0.f, 0.f}, v = k;
    if (node < n) {
      const float *kr = kb + (int64_t)node * p.k.row + 4 * c, *vr = vb + (int64_t)node * p.v.row + 4 * c;
      k = p.k_vec ? *reinterpret_cast<const f32x4*>(kr) : f32x4{kr[0], kr[1], kr[2], kr[3]};
      v = p.v_vec ? *reinterpret_cast<const f32x4*>(vr) : f32x4{vr[0], vr[1], vr[2], vr[3]};
    }
    sb[c * 16 + t] = __builtin_bit_cast(u32x4, k);
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const bool ok = is_finite(v[d]);
      odd |= !ok;
      ((float*)&sb[L::VB + 4 * (4 * c + d) + t / 4])[t % 4] = ok ? v[d] : 0.f;
    }
  }
  return odd;
}

// The (sequence, split) of work item `item`: first every split that is not its sequence's last,
// by sequence, then each sequence's last.  So the items that there are come in a row (workgroups past
// them, which end at once, would otherwise fall on some compute units and spare others) and
// the uneven ones, which take the nodes too, last.  Every wave searches by itself: 64 sequences
// at a time, a scan over the lanes.  Batches of more than kScanBatch sequences go in grid order.
constexpr int kScanBatch = 1024;

__device__ __forceinline__ bool find_item(const TreeParams& p, int item, int lane, int& b, int& s) {
  const int batch = p.st.batch;
  if (p.max_splits == 1 || batch > kScanBatch) {
    b = item / p.max_splits;
    s = item % p.max_splits;
    return true;
  }
  int base = 0;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    const int n = b0 + lane < batch ? clamp_len(p.seq_lens, b0 + lane, p.max_seq_len) : 0;
    const int full = n > 0 ? (n - 1) / p.split_len : 0;
    int sum = full;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(sum, o);
      sum += lane >= o ? v : 0;
    }
    const uint64_t past = __ballot(item < base + sum);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      b = b0 + at;
      s = item - (base + __shfl(sum, at) - __shfl(full, at));
      return true;
    }
    base += __shfl(sum, 63);
  }
  b = item - base;
  if (b >= batch) return false;
  const int n = clamp_len(p.seq_lens, b, p.max_seq_len);
  s = n > 0 ? (n - 1) / p.split_len : 0;
  return true;
}

// Partial results: each tile of 16 rows in the order in which a wave holds it, four values (16 bytes) a
// lane and side by side: o_part[tile of the split][nt][16 la + li] = dims 16 nt + 4 la .. + 3 of row li.
// So both kernels move whole lines.
__device__ __forceinline__ int64_t tile_of(const TreeParams& p, int b, int g, int s, int row0) {
  return ((((int64_t)b * p.st.n_kv + g) * p.max_splits + s) * p.r_alloc + row0) >> 4;
}

__device__ __forceinline__ float lse_of(float m, float l) {
  return l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

// One workgroup of four waves per (group of query rows, KV head; split; sequence), 16 or 32 rows a wave.
// The split's units pass through three LDS stages, loaded two units ahead, a quarter by every
// wave (a wave without rows too).  A sequence's last split takes the nodes as well, first, while its
// first units arrive.  A sequence of one split is finished here, else its splits leave (m, l) and O
// for tree_merge.
// What bounds it (8 KV heads, head dim 128).  fp32, the matrix cores: 32 sequences of 8000 tokens, 240 rows: 2090 us, 120
// TFLOP/s of 157 at the nominal clock; 4 rows, the read: 349 us, 6.0 TB/s.  Few rows, the read: 32 sequences of 131072 8-bit tokens, 4 rows each:
// 1330 us for 8.7 GB, 6.5 TB/s, where plain reads reach 7.1.  64 rows of 8-bit tokens: vector issue, most of it the
// values' conversions, one per two values and wave, and the exponentials: 128 sequences of 1K-8K: 211 us, 4.2
// TB/s and 506 TFLOP/s.  320 rows of bf16: 64 sequences of 2K-32K: 1185-1230 us with their join, 780-810
// TFLOP/s (a large library product: 1300), matrix cores 53% busy, three waves per SIMD by registers and LDS; a sixth
// of its wave slots have no rows (320 in groups of 128).  One sequence of 2048, 240 rows: 20 us, a chain of loads.
constexpr int kWaves = 4;

template <int HD, bool E8, template <int, bool> class Wave>
__global__ __launch_bounds__(64 * kWaves, 3) void tree_split(const TreeParams p) {
  using WV = Wave<HD, E8>;
  using L = typename WV::U;
  using T = typename WV::T;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int NSUB = L::NSUB, U = L::TOKENS, IPG = L::IPG, W = kWaves, NODES = WV::NODES;
  constexpr int NS = 3, D = 2;  // LDS stages, units ahead
  // A wave loads the keys and values of one run of every unit (8-bit: four runs), or its keys or values (two), or half
  // of them (fp32: one).
  constexpr int KIND = NSUB == W ? 2 : 1, LOADS = KIND * IPG + (E8 ? 1 : 0);
  static_assert(KIND * W == 2 * NSUB * L::PARTS && D * LOADS < 64, "every run once, and the loads in flight");
  static_assert(F32 || L::PIECES >= Unit<HD, false, WV::PAD>::PIECES, "a stage holds a unit of nodes");
  __shared__ u32x4 stage[NS][L::PIECES];
  __shared__ int blk_ids[2][kIdWin];
  __shared__ int odd_values[W];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  __builtin_assume(wave >= 0 && wave < W);
  const int g = blockIdx.x % p.st.n_kv, qg = blockIdx.x / p.st.n_kv;
  int b, s;
  if (!find_item(p, blockIdx.y + gridDim.y * blockIdx.z, lane, b, s)) return;
  b = __builtin_amdgcn_readfirstlane(b);
  s = __builtin_amdgcn_readfirstlane(s);
  const int n = count_of(p, b), rows = n * p.group;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len);
  const int t0 = s * p.split_len, t1 = min(len, t0 + p.split_len);
  if ((s > 0 && t0 >= len) || qg * W * WV::ROWS >= rows) return;
  const bool whole = len <= p.split_len, last = t1 == len;
  const int row0 = (qg * W + wave) * WV::ROWS;
  const bool active = row0 < rows;

  WV wv(lane);
  const int row = min(row0 + wv.row(), rows - 1), node = row / p.group, head = g * p.group + row % p.group;
  wv.load_queries((const T*)p.q.data + ((int64_t)b * p.nodes + node) * p.q.row + (int64_t)head * p.q.head, p.q_vec);

  const StoreArg& c = p.st;
  constexpr int ESZ = E8 ? 1 : sizeof(T);
  const int bs = 1 << c.bs_log2, nunits = (t1 - t0 + U - 1) / U, lastu = nunits - 1;
  const int lb0 = t0 >> c.bs_log2, nlb = t1 > t0 ? ((t1 - 1) >> c.bs_log2) - lb0 + 1 : 0;
  const int* bt_row = c.block_table ? c.block_table + (int64_t)b * c.mbps + lb0 : nullptr;
  // The first two windows of block ids and the first nodes are under way together.
  constexpr int IDS = 2 * kIdWin / (64 * W);
  static_assert(IDS * 64 * W == 2 * kIdWin, "ids per thread");
  int ids[IDS];
#pragma unroll
  for (int j = 0; j < IDS; ++j) {
    const int i = j * 64 * W + tid;
    ids[j] = !bt_row ? b * c.mbps + lb0 + i : i < nlb ? bt_row[i] : 0;
  }
  auto nodes_to_stage = [&](int u) __attribute__((always_inline)) {
    bool odd;
    if constexpr (F32) odd = stage_nodes_f32<HD, W>(p, stage[D], b, g, u, n, tid);
    else odd = stage_nodes<HD, W, WV::PAD>(p, stage[D], b, g, u, n, tid);
    const bool any = __any(odd);
    if (lane == 0) odd_values[wave] = any;
  };
  if (last) nodes_to_stage(0);
#pragma unroll
  for (int j = 0; j < IDS; ++j) (&blk_ids[0][0])[j * 64 * W + tid] = ids[j];
  auto load_window = [&](int w) __attribute__((always_inline)) {
    for (int j = wave; j < kIdWin / 64; j += W) {
      const int i = min(w * kIdWin + j * 64 + lane, nlb - 1);  // past the end: the last id again
      if (bt_row) ld4_to_lds(bt_row + i, &blk_ids[w & 1][j * 64]);
      else blk_ids[w & 1][j * 64 + lane] = b * c.mbps + lb0 + i;
    }
  };
  // This wave's run of a unit, and what it loads of it: first kind 0 keys, 1 values.
  const int run = wave * NSUB / W, kind0 = KIND == 1 ? wave & 1 : 0, part = L::PARTS == 1 ? 0 : wave >> 1;
  uint32_t lane_off[KIND];  // of the first load's pieces; the next 64 lie 64 bs bytes on (an offset for each load takes registers
                            // that waves of 32 rows lack: 1208 -> 1385 us as above)
  const char* kind_base[KIND];  // a run's place: kind_base + block * block_step + (slot << slot_shift)
  uint64_t block_step[KIND];
  int slot_shift[KIND], piece0[KIND];
  // Loads are streaming (read once by this launch), unless another query group reads the
  // same blocks, or a unit takes less than 64 bytes of a dim's row of values.
  bool stream[KIND];
  const int64_t step64 = (int64_t)64 << c.bs_log2;
#pragma unroll
  for (int k = 0; k < KIND; ++k) {
    const bool v = kind0 + k;
    lane_off[k] = v ? L::value_off(64 * IPG * part + lane, bs) : L::key_off(64 * IPG * part + lane, bs);
    kind_base[k] = v ? (const char*)c.v + g * c.v_sh * ESZ : (const char*)c.k + g * c.k_sh * ESZ;
    block_step[k] = (uint64_t)(v ? c.v_sb : c.k_sb) * ESZ;
    slot_shift[k] = v ? (E8 ? 0 : F32 ? 2 : 1) : 4;
    piece0[k] = (v ? L::VB + run * L::SUB : run * L::KP) + 64 * IPG * part;
    stream[k] = p.n_qgroups == 1 && (!v || bs * ESZ <= 64);
  }
  const uint8_t* exp_base = lane & 4 ? c.v_exp : c.k_exp;  // 8-bit: lanes 0..3 the keys' exponents, 4..7 the values'
  const uint32_t blocks = (uint32_t)(c.num_blocks < 0xffffffffll ? c.num_blocks : 0xffffffffll);
  // The next unit to issue: its number, the first token of this wave's run, and that run's block id,
  // read from LDS one unit ahead.  A run past the end reads the unit's first again.
  int next_u = 0, next_t = 0, next_id = 0;
  // When the ids read enter window w >= 1 (block ids from w * kIdWin), window w + 1 replaces w - 1,
  // which no later unit reads; kIdWin blocks later it has long landed.  (Units start at multiples
  // of 64 tokens, so no unit lies in two windows.)
  int window_end = kIdWin;
  auto look_ahead = [&]() __attribute__((always_inline)) {
    const int first = t0 + U * min(next_u, lastu);
    next_t = first + 16 * run < t1 ? first + 16 * run : first;
    const int rel = (next_t >> c.bs_log2) - lb0;
    next_id = (&blk_ids[0][0])[rel & (2 * kIdWin - 1)];
    if (rel >= window_end) {
      window_end += kIdWin;
      if (window_end < nlb) load_window(window_end / kIdWin);
    }
  };
  auto issue = [&](int buf) __attribute__((always_inline)) {
    uint32_t blk = (uint32_t)__builtin_amdgcn_readfirstlane(next_id);
    blk = blk < blocks ? blk : 0;
    const uint32_t slot = next_t & (bs - 1);
#pragma unroll
    for (int k = 0; k < KIND; ++k) {
      const char* base = kind_base[k] + blk * block_step[k] + (slot << slot_shift[k]);
      u32x4* to = &stage[buf][piece0[k]];
      if (stream[k]) {
#pragma unroll
        for (int j = 0; j < IPG; ++j) ld16_to_lds(base + j * step64, lane_off[k], to + 64 * j);
      } else {
#pragma unroll
        for (int j = 0; j < IPG; ++j) ld16_to_lds<false>(base + j * step64, lane_off[k], to + 64 * j);
      }
    }
    if constexpr (E8)
      if (lane < 8) ld4_to_lds(exp_base + blk * (uint64_t)c.e_sb + g * c.e_sh + slot + 4 * (lane & 3), &stage[buf][L::EB + 2 * run]);
    ++next_u;
    look_ahead();
  };
  // nothing that the compiler counts stays in flight past this point
  wait_vmcnt<0>();
  lds_barrier();
  if (nunits > 0) {
    look_ahead();
    issue(0);
    if (lastu > 0) issue(1);
  }
  if (last)  // the nodes, from the stage that unit D will take
    for (int u = 0; NODES * u < n; ++u) {
      if (u > 0) {
        lds_barrier();
        nodes_to_stage(u);
        lds_barrier();
      }
      if (!active) continue;
      bool odd = false;
#pragma unroll
      for (int w = 0; w < W; ++w) odd |= odd_values[w] != 0;
      const T* vb = (const T*)p.v.data + (int64_t)b * p.nodes * p.v.row + g * p.v.head;
      const uint32_t seen = seen_word(p, b, node, NODES * u / 32, n) >> (NODES * u % 32);
      // the values that are not finite, kept out of the products, reach the rows that see them alone
      wv.node_unit(stage[D], seen, p.scale_log2, odd, [&](int t, float w) {
        if (NODES * u + t >= n) return;
        const bool sees = (seen >> t) & 1;  // (a weight may have vanished: 0 times infinity is NaN, as of cached tokens)
        wv.add4([&](int d, float o) {
          const float x = to_f32(vb[(int64_t)(NODES * u + t) * p.v.row + d]);
          return sees && !is_finite(x) ? fmaf(w, x, o) : o;
        });
      });
    }
  if constexpr (E8) wv.split_queries();
  int buf = 0;
  for (int u = 0; u < nunits; ++u) {
    // this wave's loads of unit u have landed; after the barrier everyone's have, and all are past
    // unit u - 1, whose stage unit u + D takes
    if (u < lastu) wait_vmcnt<LOADS>();
    else wait_vmcnt<0>();
    lds_barrier();
    if (u + D <= lastu) issue(buf == 0 ? NS - 1 : buf - 1);
    const u32x4* sb = stage[buf];
    buf = buf == NS - 1 ? 0 : buf + 1;
    if (active) wv.cached_unit(sb, u == lastu, t1 - (t0 + U * u), p.scale_log2);
  }

  if (!active) return;
  const float l = wv.sum();
  const bool live = row0 + wv.row() < rows, first = lane < WV::ROWS;
  if (whole) {
    if (!live) return;
    if (p.lse && first) p.lse[((int64_t)b * p.nodes + node) * (p.st.n_kv * p.group) + head] = lse_of(wv.st.m, l);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    T* o = (T*)p.out.data + ((int64_t)b * p.nodes + node) * p.out.row + (int64_t)head * p.out.head;
    typedef T T4 __attribute__((ext_vector_type(4)));
    wv.each4([&](int d, f32x4 x) {
      const T4 y{from_f32<T>(x[0] * inv), from_f32<T>(x[1] * inv), from_f32<T>(x[2] * inv), from_f32<T>(x[3] * inv)};
      if (p.o_vec) *reinterpret_cast<T4*>(o + d) = y;
      else
#pragma unroll
        for (int r = 0; r < 4; ++r) o[d + r] = y[r];
    });
  } else {
    const int64_t tile = tile_of(p, b, g, s, row0 + (wv.row() & ~15));
    const int li = wv.row() & 15;
    if (first) p.ml_part[16 * tile + li] = make_float2(wv.st.m, l);
    if (live)
      wv.each4([&](int d, f32x4 x) { ((f32x4*)p.o_part)[(tile * (HD / 16) + d / 16) * 64 + d % 16 / 4 * 16 + li] = x; });
  }
}

// Joins the splits of the sequences that have several: one workgroup per tile, every split's O
// weighted by 2^(m - the largest m).  The 16 rows' weights of up to 32 splits at a time are found by
// all threads and shared through LDS.  Bound by the read of the partial results: 390 MB (64 sequences of 2K-32K
// tokens in splits of 4096, 320 rows of 8 KV heads) in 65 us, 6 TB/s.
template <int HD, typename T>
__global__ __launch_bounds__(256) void tree_merge(const TreeParams p) {
  constexpr int PER = HD / 64, CH = 32;
  __shared__ float wsh[CH][16];
  __shared__ float red[16][17];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, la = lane >> 4;
  const int row0 = 16 * blockIdx.x, g = blockIdx.y, b = blockIdx.z;
  const int len = clamp_len(p.seq_lens, b, p.max_seq_len), rows = count_of(p, b) * p.group;
  if (len <= p.split_len || row0 >= rows) return;
  const int ns = (len + p.split_len - 1) / p.split_len;
  const int r = tid & 15, c = tid >> 4;
  const float2* ml = p.ml_part + 16 * tile_of(p, b, g, 0, row0) + r;
  float m = kLowest, l = 0.f;
  for (int s = c; s < ns; s += 16) m = fmaxf(m, ml[(int64_t)s * p.r_alloc].x);
  red[r][c] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, red[r][i]);
  const bool mine = row0 + li < rows;
  const f32x4* o = (const f32x4*)p.o_part + tile_of(p, b, g, 0, row0) * (HD * 4) + tid;
  const int64_t o_split = (int64_t)p.r_alloc / 16 * (HD * 4);
  f32x4 acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < ns; s0 += CH) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < CH; j += 16) {
      const int s = s0 + c + j;
      float w = 0.f;
      if (s < ns) {
        const float2 x = ml[(int64_t)s * p.r_alloc];
        w = fast_exp2(x.x - m);
        l += w * x.y;
      }
      wsh[c + j][r] = w;
    }
    __syncthreads();
    if (!mine) continue;
    const int k1 = min(CH, ns - s0);
#pragma unroll 4
    for (int k = 0; k < k1; ++k)
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const f32x4 x = o[(s0 + k) * o_split + 256 * i];
        acc[i] += x * wsh[k][li];
      }
  }
  __syncthreads();
  red[r][c] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) l += red[r][i];
  __syncthreads();
  if (c == 0) {
    red[r][16] = l == 0.f ? 0.f : 1.0f / l;
    const int row = row0 + r;
    if (p.lse && row < rows)
      p.lse[((int64_t)b * p.nodes + row / p.group) * (p.st.n_kv * p.group) + g * p.group + row % p.group] = lse_of(m, l);
  }
  __syncthreads();
  if (!mine) return;
  const int row = row0 + li;
  const float inv = red[li][16];
  T* out = (T*)p.out.data + ((int64_t)b * p.nodes + row / p.group) * p.out.row + (int64_t)(g * p.group + row % p.group) * p.out.head;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int d = ((256 * i + tid) >> 6) * 16 + 4 * la;
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 y;
#pragma unroll
    for (int r = 0; r < 4; ++r) y[r] = from_f32<T>(acc[i][r] * inv);
    if (p.o_vec) *reinterpret_cast<T4*>(out + d) = y;
    else
#pragma unroll
      for (int r = 0; r < 4; ++r) out[d + r] = y[r];
  }
}

// ---------------------------------------------------------------- fp32
// The same rows with fp32 products, lane (li, la) as in WaveF32, for calls of few workgroups: one workgroup of 8 waves
// per (query tile, KV head; split; sequence); the waves take every eighth step of 16 tokens, cached ones and
// then, in the last split, nodes, straight from memory, and join through LDS in their order.  4 sequences of 256
// tokens, 4 nodes of 2 heads: 8 us, bound by the chain of loads, steps and join (staged through LDS, as larger calls are: 18).
constexpr int kF32Waves = 8;

template <int HD>
__global__ __launch_bounds__(64 * kF32Waves) void tree_split_f32(const TreeParams p) {
  constexpr int NJ = HD / 16, NW = kF32Waves;
  __shared__ f32x4 osh[NW][NJ][64];
  __shared__ float2 mlsh[NW][64];
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, la = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % p.st.n_kv, row0 = 16 * (blockIdx.x / p.st.n_kv);
  int b, s;
  if (!find_item(p, blockIdx.y + gridDim.y * blockIdx.z, lane, b, s)) return;
  b = __builtin_amdgcn_readfirstlane(b);
  s = __builtin_amdgcn_readfirstlane(s);
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
  float m = kLowest, l = 0.f;
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
            if (((seen >> t) & 1) && !is_finite(x)) o[j][r] = fmaf(w, x, o[j][r]);
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
    const int64_t tile = tile_of(p, b, g, s, row0);
    if (wave == 0 && la == 0) p.ml_part[16 * tile + li] = make_float2(mg, lg);
    ((f32x4*)p.o_part)[(tile * NJ + wave) * 64 + lane] = x;
  }
}

}  // namespace

hipError_t launch_tree(const TreeParams& p, int storage, int hd, hipStream_t s) {
  const int rows = p.nodes * p.group;
  hipError_t e;
  if (p.rows_per_wave == 2) {
    if (storage != SP_F32 || p.split_len % 16 || (rows + 15) / 16 * 16 > p.r_alloc) return hipErrorInvalidValue;
    const dim3 grid(p.st.n_kv * ((rows + 15) / 16), p.max_splits, p.st.batch), block(64 * kF32Waves);
    if (hd == 128) hipLaunchKernelGGL((tree_split_f32<128>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((tree_split_f32<64>), grid, block, 0, s, p);
    e = hipGetLastError();
  } else {
    if (p.split_len % 64 || p.r_alloc < rows || p.r_alloc != p.n_qgroups * p.rows_per_wave * kWaves) return hipErrorInvalidValue;
    const dim3 grid(p.st.n_kv * p.n_qgroups, p.max_splits, p.st.batch), block(64 * kWaves);
    const bool e8 = storage == SP_E4M3;
    if (storage == SP_F32) {
      if (p.rows_per_wave != 16) return hipErrorInvalidValue;
      if (hd == 128) hipLaunchKernelGGL((tree_split<128, false, WaveF32>), grid, block, 0, s, p);
      else hipLaunchKernelGGL((tree_split<64, false, WaveF32>), grid, block, 0, s, p);
    } else {
#define SP_TREE(HD_, E8_, ROWS_)                                                                   \
  if (hd == HD_ && e8 == E8_ && p.rows_per_wave == ROWS_)                                          \
    hipLaunchKernelGGL((tree_split<HD_, E8_, Wave##ROWS_>), grid, block, 0, s, p);
      if (e8 && p.rows_per_wave != 16) return hipErrorInvalidValue;
      SP_TREE(128, false, 16) SP_TREE(128, false, 32) SP_TREE(128, true, 16)
      SP_TREE(64, false, 16) SP_TREE(64, false, 32) SP_TREE(64, true, 16)
#undef SP_TREE
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess || p.max_splits == 1) return e;
  const dim3 mgrid((rows + 15) / 16, p.st.n_kv, p.st.batch), block(256);
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
