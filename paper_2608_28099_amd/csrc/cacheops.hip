// Rotary positions and the paged cache's writing and reading (include/sp_probe.h:
// sp_probe_rotary, sp_probe_cache_write, sp_probe_cache_read).  All three move every
// value once, so they are bound by memory (or, for few rows, by latency).
#include "common.h"
#include "ops.h"

namespace sp {
namespace {

struct e4m3 { uint8_t bits; };  // storage tag

// ---------------------------------------------------------------- sixteen values of a head
// A lane's 16 consecutive values as they lie in memory; `vec`: 16-byte aligned.
template <typename T>
struct Raw16 {
  u32x4 w[sizeof(T)];
};

template <typename T>
__device__ __forceinline__ Raw16<T> load_raw(const T* p, bool vec) {
  Raw16<T> x;
  if (vec) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) x.w[i] = ld16v((const char*)p + 16 * i);
  } else {
    T v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = p[i];
    __builtin_memcpy(&x, v, sizeof(x));
  }
  return x;
}

// The same of two runs of 8.
template <typename T>
__device__ __forceinline__ Raw16<T> load_raw(const T* p, const T* q, bool vec) {
  constexpr int N = sizeof(T) / 2;
  Raw16<T> x;
  if (vec) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x.w[i] = ld16v((const char*)p + 16 * i);
      x.w[N + i] = ld16v((const char*)q + 16 * i);
    }
  } else {
    T v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = i < 8 ? p[i] : q[i - 8];
    __builtin_memcpy(&x, v, sizeof(x));
  }
  return x;
}

template <typename T>
__device__ __forceinline__ void unpack(const Raw16<T>& r, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t w = r.w[i * sizeof(T) / 16][i * sizeof(T) / 4 % 4];
    x[i] = __builtin_bit_cast(float, sizeof(T) == 4 ? w : i & 1 ? w & 0xffff0000u : w << 16);
  }
}

template <typename T>
__device__ __forceinline__ void store16(T* p, bool vec, const float (&x)[16]) {
  if (vec) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = (bf16)x[8 * h + i];
        *reinterpret_cast<u32x4*>(p + 8 * h) = __builtin_bit_cast(u32x4, w);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) *reinterpret_cast<f32x4*>(p + 4 * h) = f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) p[i] = from_f32<T>(x[i]);
  }
}

// cos and sin of 2 pi x: the nearest quarter turn of x (fp64) is taken off exactly, the
// rest, at most pi / 4, goes through the Taylor sums to r^12 and r^13 (first dropped
// terms below 4e-13).
__device__ __forceinline__ void cos_sin_turns(double x, float& c, float& s) {
  const double q4 = rint(4.0 * x);
  const double r = (4.0 * x - q4) * 1.5707963267948966, z = -r * r;
  double cr = fma(1.0 / 479001600.0, z, 1.0 / 3628800.0), sr = fma(1.0 / 6227020800.0, z, 1.0 / 39916800.0);
  cr = fma(cr, z, 1.0 / 40320.0);
  sr = fma(sr, z, 1.0 / 362880.0);
  cr = fma(cr, z, 1.0 / 720.0);
  sr = fma(sr, z, 1.0 / 5040.0);
  cr = fma(cr, z, 1.0 / 24.0);
  sr = fma(sr, z, 1.0 / 120.0);
  cr = fma(cr, z, 0.5);
  sr = fma(sr, z, 1.0 / 6.0);
  cr = fma(cr, z, 1.0);
  sr = fma(sr, z, 1.0) * r;
  const int q = (int)(long long)q4 & 3;
  const float cf = (float)cr, sf = (float)sr;
  c = q == 0 ? cf : q == 1 ? -sf : q == 2 ? -cf : sf;
  s = q == 0 ? sf : q == 1 ? cf : q == 2 ? -sf : -cf;
}

// Value d of a head (d < rotary_dim), rotated: its pair's other member sits at d + half,
// d - half, d + 1 or d - 1.
struct PairOf {
  int other, pair;
  bool first;
};
__device__ __forceinline__ PairOf pair_of(int d, int rotary_dim, int layout) {
  const int half = rotary_dim >> 1;
  if (layout == SP_ROTARY_INTERLEAVED) return {d ^ 1, d >> 1, (d & 1) == 0};
  return d < half ? PairOf{d + half, d, true} : PairOf{d - half, d - half, false};
}

// ---------------------------------------------------------------- rotary
// y0 = x0 cos a - x1 sin a, y1 = x1 cos a + x0 sin a for every pair: every value read and written once, so
// bound by memory.  One workgroup per R rows: their cosines and sines once into LDS (fp64 angles), then each
// thread takes the same piece of every row, so that R rows' loads are under way together.  A pair
// is read and written by one lane, so the output may be the input.  Pieces (V values, 16
// bytes, where every head is aligned so): of interleaved heads V values of a head; of half
// heads V pairs, or V values that stay.  Else single pairs and values (kScalar).
// 16384 rows of 48 heads (half of each rotated, bf16, 403 MB): 80 us, 5.0 TB/s, where a large copy moves
// 4.8; 128 rows of 40: 3.8 us.  (Which R and pieces: rotary_typed.)
enum RotaryMode { kScalar, kHalf, kInterleaved };

template <typename T, int MODE, int R>
__global__ __launch_bounds__(256) void rotary_rows(const RotaryParams p) {
  constexpr int V = MODE == kScalar ? 1 : 16 / (int)sizeof(T);
  typedef T Piece __attribute__((ext_vector_type(V)));
  __shared__ __align__(16) float cs[R][64], sn[R][64];
  __shared__ int live[R];
  const int row0 = (blockIdx.x + gridDim.x * blockIdx.y) * R, hd = p.rot.head_dim, rd = p.rot.rotary_dim, half = rd >> 1;
  if (row0 >= p.n_rows) return;
  if ((int)threadIdx.x < R) live[threadIdx.x] = row0 + (int)threadIdx.x < p.n_rows && p.positions[row0 + threadIdx.x] >= 0;
  for (int e = threadIdx.x; e < R * half; e += 256) {
    const int r = e / half, i = e - r * half;
    if (row0 + r >= p.n_rows) break;
    float c, s;
    cos_sin_turns((double)p.positions[row0 + r] * p.rot.turns[i], c, s);
    cs[r][i] = c * p.rot.scale;
    sn[r][i] = (p.transpose ? -s : s) * p.rot.scale;
  }
  __syncthreads();
  const bool inter = MODE == kInterleaved || (MODE == kScalar && p.rot.layout == SP_ROTARY_INTERLEAVED);
  // pieces of a head: those that turn, then those that stay
  const int turn = MODE == kInterleaved ? (rd + V - 1) / V : half / V;
  const int stay0 = MODE == kInterleaved ? turn * V : rd, items = turn + (hd - stay0) / V;
  for (int e = threadIdx.x; e < (p.n_heads[0] + p.n_heads[1]) * items; e += 256) {
    const int hh = e / items, i = e - hh * items;
    const int a = hh >= p.n_heads[0] ? 1 : 0, h = a ? hh - p.n_heads[0] : hh;
    const T* x = (const T*)p.in[a].data + (int64_t)row0 * p.in[a].row + h * p.in[a].head;
    T* y = (T*)p.out[a].data + (int64_t)row0 * p.out[a].row + h * p.out[a].head;
    // first value of the piece, and of its pairs' other members
    const int d0 = i >= turn ? stay0 + (i - turn) * V : inter ? i * (MODE == kScalar ? 2 : V) : i * V;
    const int d1 = MODE == kScalar && inter ? d0 + 1 : d0 + half;
    const bool second = MODE != kInterleaved && i < turn;
    Piece u[R], w[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (live[r]) {
        u[r] = *reinterpret_cast<const Piece*>(x + r * p.in[a].row + d0);
        if (second) w[r] = *reinterpret_cast<const Piece*>(x + r * p.in[a].row + d1);
      }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (!live[r]) continue;
      if (i < turn) {
        if constexpr (MODE == kInterleaved) {
#pragma unroll
          for (int j = 0; j < V / 2; ++j) {
            const int pair = i * (V / 2) + j;
            if (pair >= half) break;  // (the last piece of a rotary_dim that V does not divide)
            const float x0 = to_f32(u[r][2 * j]), x1 = to_f32(u[r][2 * j + 1]);
            u[r][2 * j] = from_f32<T>(x0 * cs[r][pair] - x1 * sn[r][pair]);
            u[r][2 * j + 1] = from_f32<T>(x1 * cs[r][pair] + x0 * sn[r][pair]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const int pair = i * V + j;
            const float x0 = to_f32(u[r][j]), x1 = to_f32(w[r][j]);
            u[r][j] = from_f32<T>(x0 * cs[r][pair] - x1 * sn[r][pair]);
            w[r][j] = from_f32<T>(x1 * cs[r][pair] + x0 * sn[r][pair]);
          }
        }
      }
      *reinterpret_cast<Piece*>(y + r * p.out[a].row + d0) = u[r];
      if (second) *reinterpret_cast<Piece*>(y + r * p.out[a].row + d1) = w[r];
    }
  }
}

// ---------------------------------------------------------------- places
// The slot of a token, counted through the pool (block * block_size + slot), or -1.
__device__ __forceinline__ int64_t place(const StoreArg& st, int seq, int pos) {
  if (seq < 0 || seq >= st.batch || pos < 0) return -1;
  const int lb = pos >> st.bs_log2;
  if (lb >= st.mbps) return -1;
  const int64_t at = (int64_t)seq * st.mbps + lb;
  const int64_t blk = st.block_table ? (int64_t)st.block_table[at] : at;
  if (blk < 0 || blk >= st.num_blocks) return -1;
  return (blk << st.bs_log2) + (pos & ((1 << st.bs_log2) - 1));
}

// The exponent byte of a row whose largest finite magnitude is top: the smallest
// power of two with top <= 448 * 2^e = 1.75 * 2^(8 + e).
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t b = __builtin_bit_cast(uint32_t, top);
  const int e = (int)(b >> 23) - 135 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (e < -126 ? -126 : e) + 127;
}
__device__ __forceinline__ float power_of(int biased) { return __builtin_bit_cast(float, (uint32_t)biased << 23); }

// Two values to E4M3, nearest even (values within 448; anything not finite: NaN).
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, uint32_t old, bool high) {
  constexpr float kMax = 3.402823466e38f;
  a = fabsf(a) <= kMax ? a : __builtin_nanf("");
  b = fabsf(b) <= kMax ? b : __builtin_nanf("");
  return high ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, true)
              : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, false);
}

// Sixteen values in storage form.
template <typename TS> struct Stored { TS v[16]; };
template <> struct Stored<e4m3> { u32x4 w; };

template <typename TS, int LR>
__device__ __forceinline__ void pack(const float (&x)[16], Stored<TS>& out, int& biased) {
  if constexpr (sizeof(TS) == 1) {
    constexpr float kMax = 3.402823466e38f;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float a = fabsf(x[i]);
      top = fmaxf(top, a <= kMax ? a : 0.f);
    }
#pragma unroll
    for (int o = 1; o < LR; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));  // the row's LR lanes
    biased = exponent_of(top);
    const float f = power_of(254 - biased);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t v = to_e4m3(x[4 * w] * f, x[4 * w + 1] * f, 0, false);
      out.w[w] = to_e4m3(x[4 * w + 2] * f, x[4 * w + 3] * f, v, true);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) out.v[i] = from_f32<TS>(x[i]);
  }
}

// ---------------------------------------------------------------- write
// Workgroups per tile of 64 rows: one for the values of each KV head, one for the keys of every
// heads_per_wg heads.  Keys go straight from registers: 16 values are one, two or four
// pieces of the paged layout, and eight rows of a wave that follow one another in a block make
// 128 consecutive bytes of each piece; their angles' cosines and sines are found once for all
// of the workgroup's heads.  Values lie dim-major in the cache, so they pass through LDS: where the rows of
// a tile fill an aligned group of 16 bytes' worth of slots (a "group": 4, 8 or 16 rows that
// follow one another), each dim of it is one 16-byte store; what is left, at a run's
// ends or with scattered rows, is stored value by value.
// 49152 rows of 8 heads (bf16 rows, head dim 128) of one sequence from position 0, where every group is whole: 8-bit 61 us
// (302 MB, 4.9 TB/s), with a rotation 87 (the angles, and four heads in turn); bf16 94 us (403 MB, 4.3 TB/s), rotated 97.
// Tiles are cut by rows: of a sequence whose first row and slot differ modulo X each tile's end cuts a group, of 8-bit
// rows a quarter, which goes value by value.  16 sequences of 2K-4K tokens, 44377 rows in all, 8-bit, rotated: 113 us (273 MB, 2.4
// TB/s).  128 rows: 4.4 to 4.9 us, rotated 8.4 to 9.
constexpr int kTile = 64;

struct TilePlan {
  int64_t dest[kTile];
  int src[kTile];
  int lead[kTile], single[kTile];  // first rows of whole groups; rows outside them
  int n_lead, n_single;
};

// By the first wave: rows row0 .. of the tile, X slots per group.
template <int X>
__device__ __forceinline__ void plan_tile(const CacheParams& p, int row0, TilePlan& t) {
  const int r = threadIdx.x;
  int64_t d = -1;
  int src = 0;
  if (row0 + r < p.n_rows) {
    src = row0 + r;
    if (p.src) src = p.src[row0 + r];
    d = place(p.st, p.seq_ids[row0 + r], p.positions[row0 + r]);
    if (src < 0 || src >= p.n_src) d = -1;
  }
  t.dest[r] = d;
  t.src[r] = src;
  // a group starts at a slot that is a multiple of X and takes the next X - 1 rows
  const int64_t next = __shfl_down(d, 1);
  const bool follows = r < kTile - 1 && d >= 0 && next == d + 1;
  const uint64_t chain = __ballot(follows);                     // row r + 1 is the next slot
  const uint64_t want = ((1ull << (X - 1)) - 1);
  const bool lead = d >= 0 && (d & (X - 1)) == 0 && r + X <= kTile && ((chain >> r) & want) == want;
  const uint64_t leads = __ballot(lead);
  // covered: some leader among rows r - X + 1 .. r
  const int lo = r >= X - 1 ? r - (X - 1) : 0;
  const uint64_t upto = r == 63 ? ~0ull : ((1ull << (r + 1)) - 1);
  const bool covered = ((leads & upto) >> lo) != 0;
  const bool single = d >= 0 && !covered;
  const uint64_t singles = __ballot(single), below = (1ull << r) - 1;
  if (lead) t.lead[__popcll(leads & below)] = r;
  if (single) t.single[__popcll(singles & below)] = r;
  if (r == 0) {
    t.n_lead = __popcll(leads);
    t.n_single = __popcll(singles);
  }
}

// How keys are rotated.  kHalf8: half layout, rotary_dim / 2 a multiple of 8: a lane takes two runs of 8
// values that pair with each other; kPairs: interleaved, pairs within the lane's 16; kAny: any half layout.
enum KeyRotation { kNoRotation, kHalf8, kPairs, kAny };

template <typename TS, typename TI, int HD, int ROT>
__global__ __launch_bounds__(256) void cache_write(const CacheParams p, const sp_rotary rot) {
  constexpr int LR = HD / 16, RP = 256 / LR, X = 16 / sizeof(TS);
  constexpr int VP = kTile + 4 / sizeof(TS);  // pitch of a dim's row of values
  constexpr int TP = HD / 2 + 4;              // pitch of a row's cosines (rows on different banks)
  constexpr size_t kTrig = ROT == kNoRotation ? 16 : 2 * RP * TP * sizeof(float), kValues = HD * VP * sizeof(TS);
  __shared__ TilePlan t;
  __shared__ __align__(16) char lds[kTrig > kValues ? kTrig : kValues];
  const int tid = threadIdx.x, row0 = blockIdx.x * kTile;
  const int64_t bs = (int64_t)1 << p.st.bs_log2;
  const int c = tid % LR, d0 = 16 * c;
  if (tid < kTile) plan_tile<X>(p, row0, t);
  __syncthreads();
  if ((int)blockIdx.y >= p.st.n_kv) {  // keys
    float* cs = (float*)lds;
    float* sn = cs + RP * TP;
    const int h0 = ((int)blockIdx.y - p.st.n_kv) * p.heads_per_wg, h1 = min(h0 + p.heads_per_wg, p.st.n_kv);
    const int rd = rot.rotary_dim, half = rd >> 1;
    // first values of the lane's two runs of 8 (which lie side by side but for the pairs of kHalf8)
    const bool turns = ROT == kHalf8 && d0 < rd;
    const int da = turns ? 8 * c : d0, db = turns ? half + 8 * c : d0 + 8;
    for (int r0 = 0; r0 < kTile; r0 += RP) {
      const int rr = tid / LR, r = r0 + rr;
      const int64_t dest = t.dest[r];
      const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
      const TI* kr = (const TI*)p.k.data + (int64_t)t.src[r] * p.k.row;
      // the next head's values are under way while this one's are rotated, packed and stored
      Raw16<TI> x;
      if (dest >= 0) x = load_raw(kr + h0 * p.k.head + da, kr + h0 * p.k.head + db, p.k_vec);
      if constexpr (ROT != kNoRotation) {
        if (r0) __syncthreads();
        for (int e = tid; e < RP * half; e += 256) {
          const int q = e / half, i = e - q * half;
          if (t.dest[r0 + q] < 0) continue;
          float co, si;
          cos_sin_turns((double)p.positions[row0 + r0 + q] * rot.turns[i], co, si);
          cs[q * TP + i] = co * rot.scale;
          sn[q * TP + i] = si * rot.scale;
        }
        __syncthreads();
      }
      if (dest < 0) continue;  // (the LR lanes of a row alike)
      const float* co = cs + rr * TP;
      const float* si = sn + rr * TP;
      for (int h = h0; h < h1; ++h) {
        Raw16<TI> x1;
        if (h + 1 < h1) x1 = load_raw(kr + (h + 1) * p.k.head + da, kr + (h + 1) * p.k.head + db, p.k_vec);
        float k[16];
        unpack(x, k);
        if constexpr (ROT == kHalf8) {
          if (turns)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float a = k[i], b = k[8 + i], cc = co[da + i], ss = si[da + i];
              k[i] = a * cc - b * ss;
              k[8 + i] = b * cc + a * ss;
            }
        } else if constexpr (ROT == kPairs) {
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            if (d0 + i >= rd) continue;
            const float a = k[i], b = k[i + 1], cc = co[d0 / 2 + i / 2], ss = si[d0 / 2 + i / 2];
            k[i] = a * cc - b * ss;
            k[i + 1] = b * cc + a * ss;
          }
        } else if constexpr (ROT == kAny) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (d0 + i >= rd) continue;
            const PairOf o = pair_of(d0 + i, rd, rot.layout);
            const float z = to_f32(kr[h * p.k.head + o.other]);
            k[i] = o.first ? k[i] * co[o.pair] - z * si[o.pair] : k[i] * co[o.pair] + z * si[o.pair];
          }
        }
        Stored<TS> w;
        int biased = 0;
        pack<TS, LR>(k, w, biased);
        TS* kb = (TS*)p.st.k + blk * p.st.k_sb + h * p.st.k_sh;
        if constexpr (sizeof(TS) == 1) {
          if constexpr (ROT == kHalf8) {
            *reinterpret_cast<u32x2*>(kb + ((int64_t)(da / X) * bs + slot) * X + da % X) = u32x2{w.w[0], w.w[1]};
            *reinterpret_cast<u32x2*>(kb + ((int64_t)(db / X) * bs + slot) * X + db % X) = u32x2{w.w[2], w.w[3]};
          } else {
            *reinterpret_cast<u32x4*>(kb + ((int64_t)c * bs + slot) * X) = w.w;
          }
          if (c == 0) p.st.k_exp[blk * p.st.e_sb + h * p.st.e_sh + slot] = (uint8_t)biased;
        } else {
#pragma unroll
          for (int q = 0; q < 16 / X; ++q) {
            const int d = q < 8 / X ? da + q * X : db + (q - 8 / X) * X;
            u32x4 piece;
            __builtin_memcpy(&piece, &w.v[q * X], 16);
            *reinterpret_cast<u32x4*>(kb + ((int64_t)(d / X) * bs + slot) * X) = piece;
          }
        }
        x = x1;
      }
    }
    return;
  }
  // values
  TS* vt = (TS*)lds;
  const int h = blockIdx.y;
  for (int r = tid / LR; r < kTile; r += RP) {
    const int64_t dest = t.dest[r];
    if (dest < 0) continue;
    const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
    float x[16];
    Stored<TS> w;
    int biased = 0;
    unpack(load_raw((const TI*)p.v.data + (int64_t)t.src[r] * p.v.row + h * p.v.head + d0, p.v_vec), x);
    pack<TS, LR>(x, w, biased);
    if constexpr (sizeof(TS) == 1) {
      if (c == 0) p.st.v_exp[blk * p.st.e_sb + h * p.st.e_sh + slot] = (uint8_t)biased;
#pragma unroll
      for (int i = 0; i < 16; ++i) vt[(d0 + i) * VP + r].bits = (uint8_t)(w.w[i / 4] >> (8 * (i % 4)));
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) vt[(d0 + i) * VP + r] = w.v[i];
    }
  }
  __syncthreads();
  const int nl = t.n_lead, ns = t.n_single;
  for (int e = tid; e < nl * HD; e += 256) {
    const int d = e / nl, r = t.lead[e - d * nl];
    const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
    TS piece[X];
#pragma unroll
    for (int i = 0; i < X; ++i) piece[i] = vt[d * VP + r + i];
    u32x4 w;
    __builtin_memcpy(&w, piece, 16);
    *reinterpret_cast<u32x4*>((TS*)p.st.v + blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot) = w;
  }
  for (int e = tid; e < ns * HD; e += 256) {
    const int r = t.single[e / HD], d = e % HD;
    const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
    ((TS*)p.st.v)[blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot] = vt[d * VP + r];
  }
}

// ---------------------------------------------------------------- read
// The same tiles the other way, a workgroup per KV head for the keys and one for the values: values
// through LDS, by groups where the tokens make them, word by word.  49152 rows of 8 heads to bf16
// (head dim 128) where every group is whole: from 8-bit 70 us (302 MB, 4.3 TB/s; byte by byte through LDS 79), from bf16 79
// (403 MB, 5.1 TB/s; 82).  32 sequences of 1K-4K 8-bit tokens, 69773 rows in all, a quarter of them outside groups: 121 us (430 MB,
// 3.5 TB/s).  Scattered tokens, whose values lie a byte or two apart: 158 and 324.  More heads a workgroup gain
// nothing (8-bit: 71, 76, 77, 88 us with 1, 2, 4, 8).
template <typename TS>
__device__ __forceinline__ float value_of(TS x) {
  if constexpr (sizeof(TS) == 1) return __builtin_amdgcn_cvt_f32_fp8((int)x.bits, 0);
  else return to_f32(x);
}

template <typename T>
__device__ __forceinline__ void store8(T* p, bool vec, const float (&x)[8]) {
  if (vec) {
    if constexpr (sizeof(T) == 2) {
      bf16x8 w;
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = (bf16)x[i];
      *reinterpret_cast<u32x4*>(p) = __builtin_bit_cast(u32x4, w);
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) *reinterpret_cast<f32x4*>(p + 4 * h) = f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = from_f32<T>(x[i]);
  }
}

template <typename TS, typename TI, int HD>
__global__ __launch_bounds__(256) void cache_read(const CacheParams p) {
  constexpr int LR = HD / 16, RP = 256 / LR, X = 16 / sizeof(TS);
  constexpr int Q = 4 / sizeof(TS);  // values of a word
  constexpr int VP = kTile + Q;      // pitch of a dim's row of values, a whole number of words
  __shared__ TilePlan t;
  __shared__ __align__(16) TS vt[HD * VP];
  const int tid = threadIdx.x, row0 = blockIdx.x * kTile;
  const int64_t bs = (int64_t)1 << p.st.bs_log2;
  const bool keys = p.k.data && (int)blockIdx.y < p.st.n_kv;
  const int h = blockIdx.y % p.st.n_kv;
  if (tid < kTile) plan_tile<X>(p, row0, t);
  __syncthreads();
  if (keys) {
    const int c = tid % LR, d0 = 16 * c;
    for (int r = tid / LR; r < kTile; r += RP) {
      const int64_t dest = t.dest[r];
      if (dest < 0) continue;
      const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1), row = row0 + r;
      float x[16], f = 1.f;
      if constexpr (sizeof(TS) == 1) f = power_of(p.st.k_exp[blk * p.st.e_sb + h * p.st.e_sh + slot]);
      const TS* kb = (const TS*)p.st.k + blk * p.st.k_sb + h * p.st.k_sh;
#pragma unroll
      for (int q = 0; q < 16 / X; ++q) {
        const u32x4 w = ld16v(kb + ((int64_t)(c * (16 / X) + q) * bs + slot) * X);
        TS piece[X];
        __builtin_memcpy(piece, &w, 16);
#pragma unroll
        for (int i = 0; i < X; ++i) x[q * X + i] = value_of(piece[i]) * f;
      }
      store16((TI*)p.k.data + row * p.k.row + h * p.k.head + d0, p.k_vec, x);
    }
    return;
  }
  const int nl = t.n_lead, ns = t.n_single;
  for (int e = tid; e < nl * HD; e += 256) {
    const int d = e / nl, r = t.lead[e - d * nl];
    const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
    const u32x4 w = ld16v((const TS*)p.st.v + blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot);
    if (r % Q == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(vt + d * VP + r)[i] = w[i];
    } else {
      TS piece[X];
      __builtin_memcpy(piece, &w, 16);
#pragma unroll
      for (int i = 0; i < X; ++i) vt[d * VP + r + i] = piece[i];
    }
  }
  for (int e = tid; e < ns * HD; e += 256) {
    const int r = t.single[e / HD], d = e % HD;
    const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
    vt[d * VP + r] = ((const TS*)p.st.v)[blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot];
  }
  __syncthreads();
  // a lane takes 8 dims of the Q rows whose values share words
  for (int e = tid; e < kTile / Q * (HD / 8); e += 256) {
    const int d0 = 8 * (e % (HD / 8)), r0 = Q * (e / (HD / 8));
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = *reinterpret_cast<const uint32_t*>(vt + (d0 + i) * VP + r0);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int64_t dest = t.dest[r0 + q];
      if (dest < 0) continue;
      const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1), row = row0 + r0 + q;
      float x[8], f = 1.f;
      if constexpr (sizeof(TS) == 1) f = power_of(p.st.v_exp[blk * p.st.e_sb + h * p.st.e_sh + slot]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        TS part[Q];
        __builtin_memcpy(part, &w[i], 4);
        x[i] = value_of(part[q]) * f;
      }
      store8((TI*)p.v.data + row * p.v.row + h * p.v.head + d0, p.v_vec, x);
    }
  }
}

template <typename TS, typename TI, int HD>
hipError_t write_hd(const CacheParams& p, dim3 grid, hipStream_t s) {
  const sp_rotary none{};
  CacheParams d = p;
  d.rot = nullptr;
  const dim3 block(256);
  if (!p.rot) hipLaunchKernelGGL((cache_write<TS, TI, HD, kNoRotation>), grid, block, 0, s, d, none);
  else if (p.rot->layout == SP_ROTARY_HALF && p.rot->rotary_dim % 16 == 0)
    hipLaunchKernelGGL((cache_write<TS, TI, HD, kHalf8>), grid, block, 0, s, d, *p.rot);
  else if (p.rot->layout == SP_ROTARY_INTERLEAVED)
    hipLaunchKernelGGL((cache_write<TS, TI, HD, kPairs>), grid, block, 0, s, d, *p.rot);
  else hipLaunchKernelGGL((cache_write<TS, TI, HD, kAny>), grid, block, 0, s, d, *p.rot);
  return hipGetLastError();
}

template <typename TS, typename TI>
hipError_t write_typed(const CacheParams& p, int hd, dim3 grid, hipStream_t s) {
  return hd == 128 ? write_hd<TS, TI, 128>(p, grid, s) : write_hd<TS, TI, 64>(p, grid, s);
}

template <typename TS, typename TI>
hipError_t read_typed(const CacheParams& p, int hd, dim3 grid, hipStream_t s) {
  if (hd == 128) hipLaunchKernelGGL((cache_read<TS, TI, 128>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((cache_read<TS, TI, 64>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

// KV heads of a workgroup of keys: one, or with a rotation up to four that leave a workgroup per compute
// unit (their angles are found once, but their rows pass one after the other).  Rows of 8 heads, bf16 and
// 8-bit, in us with 1 / 2 / 4 / 8 heads a workgroup: 2048 rows 10.7 / 11.2 / 13.0 / 16.9 and 10.9 / 12.1 / 15.2 / 21.6; 8192 rows
// 27.2 / 19.7 / 19.9 / 24.8 and 26.0 / 22.4 / 20.1 / 27.3; 49152 rows 124 / 105 / 98 / 104 and 119 / 96 / 87 / 86.
int heads_per_wg(const CacheParams& p, int n_cus) {
  if (!p.rot) return 1;
  const int64_t tiles = (p.n_rows + kTile - 1) / kTile;
  int hpw = p.st.n_kv < 4 ? p.st.n_kv : 4;
  while (hpw > 1 && tiles * ((p.st.n_kv + hpw - 1) / hpw) < n_cus) hpw = (hpw + 1) / 2;
  return hpw;
}

// 16-byte pieces where alignment allows them (bf16, 48 heads, half of each turned: 128 rows 4.5 us, in
// single values 11.6; 16384 rows 80 and 165).  One row a workgroup, but four of interleaved
// heads where that leaves four workgroups per compute unit (40 heads, 16384 rows: 75 us with one, 66 with four; 1024 rows 6.4 and
// 7.8; half heads, 16384 rows: 61 and 65).
template <typename T>
hipError_t rotary_typed(const RotaryParams& p, int n_cus, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  // a dimension of a launch has less than 2^32 threads: groups of rows past kAcross go on in the grid's second one
  constexpr int kAcross = 1 << 23;
  auto grid = [](int groups) { return dim3(groups < kAcross ? groups : kAcross, (groups + kAcross - 1) / kAcross); };
  const dim3 block(256);
  if (p.vec && p.rot.layout == SP_ROTARY_INTERLEAVED) {
    constexpr int R = 4;
    if (p.n_rows >= 4 * R * n_cus)
      hipLaunchKernelGGL((rotary_rows<T, kInterleaved, R>), grid((p.n_rows + R - 1) / R), block, 0, s, p);
    else hipLaunchKernelGGL((rotary_rows<T, kInterleaved, 1>), grid(p.n_rows), block, 0, s, p);
  } else if (p.vec && p.rot.rotary_dim % (2 * V) == 0) {
    hipLaunchKernelGGL((rotary_rows<T, kHalf, 1>), grid(p.n_rows), block, 0, s, p);
  } else {
    hipLaunchKernelGGL((rotary_rows<T, kScalar, 1>), grid(p.n_rows), block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, int bf16_rows, int n_cus, hipStream_t s) {
  if (p.n_rows <= 0) return hipSuccess;
  return bf16_rows ? rotary_typed<bf16>(p, n_cus, s) : rotary_typed<float>(p, n_cus, s);
}

hipError_t launch_cache_write(const CacheParams& p0, int storage, int bf16_rows, int hd, int n_cus, hipStream_t s) {
  if (p0.n_rows <= 0) return hipSuccess;
  CacheParams p = p0;
  p.heads_per_wg = heads_per_wg(p, n_cus);
  const dim3 grid((p.n_rows + kTile - 1) / kTile, p.st.n_kv + (p.st.n_kv + p.heads_per_wg - 1) / p.heads_per_wg);
  switch (storage) {
    case SP_F32: return bf16_rows ? write_typed<float, bf16>(p, hd, grid, s) : write_typed<float, float>(p, hd, grid, s);
    case SP_BF16: return bf16_rows ? write_typed<bf16, bf16>(p, hd, grid, s) : write_typed<bf16, float>(p, hd, grid, s);
    case SP_E4M3: return bf16_rows ? write_typed<e4m3, bf16>(p, hd, grid, s) : write_typed<e4m3, float>(p, hd, grid, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_cache_read(const CacheParams& p, int storage, int bf16_rows, int hd, hipStream_t s) {
  if (p.n_rows <= 0) return hipSuccess;
  const dim3 grid((p.n_rows + kTile - 1) / kTile, p.st.n_kv * ((p.k.data != nullptr) + (p.v.data != nullptr)));
  switch (storage) {
    case SP_F32: return bf16_rows ? read_typed<float, bf16>(p, hd, grid, s) : read_typed<float, float>(p, hd, grid, s);
    case SP_BF16: return bf16_rows ? read_typed<bf16, bf16>(p, hd, grid, s) : read_typed<bf16, float>(p, hd, grid, s);
    case SP_E4M3: return bf16_rows ? read_typed<e4m3, bf16>(p, hd, grid, s) : read_typed<e4m3, float>(p, hd, grid, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace sp
