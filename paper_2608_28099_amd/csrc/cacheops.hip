// Rotary positions and the paged cache's writing and reading (include/sp_probe.h:
// sp_probe_rotary, sp_probe_cache_write, sp_probe_cache_read).  All three move every
// value once, so they are bound by memory (or, for few rows, by latency).
#include "common.h"
#include "ops.h"

namespace sp {
namespace {

struct e4m3 { uint8_t bits; };  // storage tag

// ---------------------------------------------------------------- sixteen values of a head
// The lane's 16 consecutive values in fp32; `vec`: 16-byte aligned.
template <typename T>
__device__ __forceinline__ void load16(const T* p, bool vec, float (&x)[16]) {
  if (vec) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 w = __builtin_bit_cast(bf16x8, ld16v(p + 8 * h));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * h + i] = (float)w[i];
      }
    } else {
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const f32x4 w = *reinterpret_cast<const f32x4*>(p + 4 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * h + i] = w[i];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = to_f32(p[i]);
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
// One workgroup per row: the row's cosines and sines once into LDS, then every value
// of every head.  A pair is read and written by one lane, so the output may be the
// input.
template <typename T>
__global__ __launch_bounds__(256) void rotary_rows(const RotaryParams p) {
  __shared__ float cs[64], sn[64];
  const int row = blockIdx.x, hd = p.rot.head_dim, rd = p.rot.rotary_dim, half = rd >> 1;
  const int pos = p.positions[row];
  if (pos < 0) return;
  if ((int)threadIdx.x < half) {
    float c, s;
    cos_sin_turns((double)pos * p.rot.turns[threadIdx.x], c, s);
    cs[threadIdx.x] = c * p.rot.scale;
    sn[threadIdx.x] = (p.transpose ? -s : s) * p.rot.scale;
  }
  __syncthreads();
  const int items = half + hd - rd;  // pairs, then the values that stay
  for (int a = 0; a < 2; ++a) {
    const T* x = (const T*)p.in[a].data + (int64_t)row * p.in[a].row;
    T* y = (T*)p.out[a].data + (int64_t)row * p.out[a].row;
    for (int e = threadIdx.x; e < p.n_heads[a] * items; e += 256) {
      const int h = e / items, i = e % items;
      const T* xh = x + h * p.in[a].head;
      T* yh = y + h * p.out[a].head;
      if (i < half) {
        const int d0 = p.rot.layout == SP_ROTARY_INTERLEAVED ? 2 * i : i;
        const int d1 = pair_of(d0, rd, p.rot.layout).other;
        const float x0 = to_f32(xh[d0]), x1 = to_f32(xh[d1]);
        yh[d0] = from_f32<T>(x0 * cs[i] - x1 * sn[i]);
        yh[d1] = from_f32<T>(x1 * cs[i] + x0 * sn[i]);
      } else {
        yh[rd + i - half] = xh[rd + i - half];
      }
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
// One workgroup per (tile of 64 rows, heads_per_wg KV heads).  Keys go straight from
// registers: 16 values are one, two or four pieces of the paged layout, and eight rows of
// a wave that follow one another in a block make 128 consecutive bytes of each piece.
// Values lie dim-major in the cache, so they pass through LDS: where the rows of a tile
// fill an aligned group of 16 bytes' worth of slots (a "group": 4, 8 or 16 rows that
// follow one another), each dim of it is one 16-byte store; what is left, at a run's
// ends or with scattered rows, is stored value by value.
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

template <typename TS, typename TI, int HD, bool ROT>
__global__ __launch_bounds__(256) void cache_write(const CacheParams p, const sp_rotary rot) {
  constexpr int LR = HD / 16, RP = 256 / LR, X = 16 / sizeof(TS);
  constexpr int VP = kTile + 4 / sizeof(TS);  // pitch of a dim's row of values
  __shared__ TilePlan t;
  __shared__ TS vt[HD * VP];
  __shared__ float cs[ROT ? kTile * 64 : 1], sn[ROT ? kTile * 64 : 1];
  const int tid = threadIdx.x, row0 = blockIdx.x * kTile;
  const int h0 = blockIdx.y * p.heads_per_wg, h1 = min(h0 + p.heads_per_wg, p.st.n_kv);
  const int64_t bs = (int64_t)1 << p.st.bs_log2;
  if (tid < kTile) plan_tile<X>(p, row0, t);
  __syncthreads();
  if constexpr (ROT) {
    const int half = rot.rotary_dim >> 1;
    for (int e = tid; e < kTile * half; e += 256) {
      const int r = e / half, i = e % half;
      if (t.dest[r] < 0) continue;
      float c, s;
      cos_sin_turns((double)p.positions[row0 + r] * rot.turns[i], c, s);
      cs[r * 64 + i] = c * rot.scale;
      sn[r * 64 + i] = s * rot.scale;
    }
    __syncthreads();
  }
  for (int h = h0; h < h1; ++h) {
    for (int r = tid / LR; r < kTile; r += RP) {
      const int c = tid % LR, d0 = 16 * c;
      const int64_t dest = t.dest[r];
      if (dest < 0) continue;  // (the LR lanes of a row alike)
      const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
      float x[16];
      const TI* kr = (const TI*)p.k.data + (int64_t)t.src[r] * p.k.row + h * p.k.head;
      load16(kr + d0, p.k_vec, x);
      if constexpr (ROT) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int d = d0 + i;
          if (d >= rot.rotary_dim) continue;
          const PairOf o = pair_of(d, rot.rotary_dim, rot.layout);
          const float y = to_f32(kr[o.other]), co = cs[r * 64 + o.pair], si = sn[r * 64 + o.pair];
          x[i] = o.first ? x[i] * co - y * si : x[i] * co + y * si;
        }
      }
      Stored<TS> w;
      int biased = 0;
      pack<TS, LR>(x, w, biased);
      TS* kb = (TS*)p.st.k + blk * p.st.k_sb + h * p.st.k_sh;
      if constexpr (sizeof(TS) == 1) {
        *reinterpret_cast<u32x4*>(kb + ((int64_t)c * bs + slot) * X) = w.w;
        if (c == 0) p.st.k_exp[blk * p.st.e_sb + h * p.st.e_sh + slot] = (uint8_t)biased;
      } else {
#pragma unroll
        for (int q = 0; q < 16 / X; ++q) {
          u32x4 piece;
          __builtin_memcpy(&piece, &w.v[q * X], 16);
          *reinterpret_cast<u32x4*>(kb + ((int64_t)(c * (16 / X) + q) * bs + slot) * X) = piece;
        }
      }
      load16((const TI*)p.v.data + (int64_t)t.src[r] * p.v.row + h * p.v.head + d0, p.v_vec, x);
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
      const int r = t.lead[e % nl], d = e / nl;
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
    __syncthreads();
  }
}

// ---------------------------------------------------------------- read
// The same tiles the other way: values through LDS, by groups where the tokens make them.
template <typename TS>
__device__ __forceinline__ float value_of(TS x) {
  if constexpr (sizeof(TS) == 1) return __builtin_amdgcn_cvt_f32_fp8((int)x.bits, 0);
  else return to_f32(x);
}

template <typename TS, typename TI, int HD>
__global__ __launch_bounds__(256) void cache_read(const CacheParams p) {
  constexpr int LR = HD / 16, RP = 256 / LR, X = 16 / sizeof(TS);
  constexpr int VP = kTile + 4 / sizeof(TS);
  __shared__ TilePlan t;
  __shared__ TS vt[HD * VP];
  const int tid = threadIdx.x, row0 = blockIdx.x * kTile;
  const int h0 = blockIdx.y * p.heads_per_wg, h1 = min(h0 + p.heads_per_wg, p.st.n_kv);
  const int64_t bs = (int64_t)1 << p.st.bs_log2;
  if (tid < kTile) plan_tile<X>(p, row0, t);
  __syncthreads();
  const int nl = t.n_lead, ns = t.n_single;
  for (int h = h0; h < h1; ++h) {
    if (p.v.data) {
      for (int e = tid; e < nl * HD; e += 256) {
        const int r = t.lead[e % nl], d = e / nl;
        const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
        const u32x4 w = ld16v((const TS*)p.st.v + blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot);
        TS piece[X];
        __builtin_memcpy(piece, &w, 16);
#pragma unroll
        for (int i = 0; i < X; ++i) vt[d * VP + r + i] = piece[i];
      }
      for (int e = tid; e < ns * HD; e += 256) {
        const int r = t.single[e / HD], d = e % HD;
        const int64_t dest = t.dest[r], blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
        vt[d * VP + r] = ((const TS*)p.st.v)[blk * p.st.v_sb + h * p.st.v_sh + d * bs + slot];
      }
    }
    __syncthreads();
    for (int r = tid / LR; r < kTile; r += RP) {
      const int c = tid % LR, d0 = 16 * c;
      const int64_t dest = t.dest[r];
      if (dest < 0) continue;
      const int64_t blk = dest >> p.st.bs_log2, slot = dest & (bs - 1);
      const int64_t row = row0 + r;
      float x[16];
      if (p.k.data) {
        const TS* kb = (const TS*)p.st.k + blk * p.st.k_sb + h * p.st.k_sh;
        float f = 1.f;
        if constexpr (sizeof(TS) == 1) f = power_of(p.st.k_exp[blk * p.st.e_sb + h * p.st.e_sh + slot]);
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
      if (p.v.data) {
        float f = 1.f;
        if constexpr (sizeof(TS) == 1) f = power_of(p.st.v_exp[blk * p.st.e_sb + h * p.st.e_sh + slot]);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = value_of(vt[(d0 + i) * VP + r]) * f;
        store16((TI*)p.v.data + row * p.v.row + h * p.v.head + d0, p.v_vec, x);
      }
    }
    __syncthreads();
  }
}

template <typename TS, typename TI>
hipError_t write_typed(const CacheParams& p, int hd, dim3 grid, hipStream_t s) {
  const sp_rotary none{};
  const sp_rotary& r = p.rot ? *p.rot : none;
  CacheParams d = p;
  d.rot = nullptr;
  if (hd == 128) {
    if (p.rot) hipLaunchKernelGGL((cache_write<TS, TI, 128, true>), grid, dim3(256), 0, s, d, r);
    else hipLaunchKernelGGL((cache_write<TS, TI, 128, false>), grid, dim3(256), 0, s, d, r);
  } else {
    if (p.rot) hipLaunchKernelGGL((cache_write<TS, TI, 64, true>), grid, dim3(256), 0, s, d, r);
    else hipLaunchKernelGGL((cache_write<TS, TI, 64, false>), grid, dim3(256), 0, s, d, r);
  }
  return hipGetLastError();
}

template <typename TS, typename TI>
hipError_t read_typed(const CacheParams& p, int hd, dim3 grid, hipStream_t s) {
  if (hd == 128) hipLaunchKernelGGL((cache_read<TS, TI, 128>), grid, dim3(256), 0, s, p);
  else hipLaunchKernelGGL((cache_read<TS, TI, 64>), grid, dim3(256), 0, s, p);
  return hipGetLastError();
}

// KV heads per workgroup: as many as leave two workgroups per compute unit (the places and
// the angles of a tile are found once for all of them).
int heads_per_wg(const CacheParams& p, int n_cus) {
  const int64_t tiles = (p.n_rows + kTile - 1) / kTile;
  int hpw = p.st.n_kv;
  while (hpw > 1 && tiles * ((p.st.n_kv + hpw - 1) / hpw) < 2 * (int64_t)n_cus) hpw = (hpw + 1) / 2;
  return hpw;
}

}  // namespace

hipError_t launch_rotary(const RotaryParams& p, int bf16_rows, int n_cus, hipStream_t s) {
  (void)n_cus;
  if (p.n_rows <= 0) return hipSuccess;
  const dim3 grid(p.n_rows), block(256);
  if (bf16_rows) hipLaunchKernelGGL((rotary_rows<bf16>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((rotary_rows<float>), grid, block, 0, s, p);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheParams& p0, int storage, int bf16_rows, int hd, int n_cus, hipStream_t s) {
  if (p0.n_rows <= 0) return hipSuccess;
  CacheParams p = p0;
  p.heads_per_wg = heads_per_wg(p, n_cus);
  const dim3 grid((p.n_rows + kTile - 1) / kTile, (p.st.n_kv + p.heads_per_wg - 1) / p.heads_per_wg);
  switch (storage) {
    case SP_F32: return bf16_rows ? write_typed<float, bf16>(p, hd, grid, s) : write_typed<float, float>(p, hd, grid, s);
    case SP_BF16: return bf16_rows ? write_typed<bf16, bf16>(p, hd, grid, s) : write_typed<bf16, float>(p, hd, grid, s);
    case SP_E4M3: return bf16_rows ? write_typed<e4m3, bf16>(p, hd, grid, s) : write_typed<e4m3, float>(p, hd, grid, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_cache_read(const CacheParams& p0, int storage, int bf16_rows, int hd, int n_cus, hipStream_t s) {
  if (p0.n_rows <= 0) return hipSuccess;
  CacheParams p = p0;
  p.heads_per_wg = heads_per_wg(p, n_cus);
  const dim3 grid((p.n_rows + kTile - 1) / kTile, (p.st.n_kv + p.heads_per_wg - 1) / p.heads_per_wg);
  switch (storage) {
    case SP_F32: return bf16_rows ? read_typed<float, bf16>(p, hd, grid, s) : read_typed<float, float>(p, hd, grid, s);
    case SP_BF16: return bf16_rows ? read_typed<bf16, bf16>(p, hd, grid, s) : read_typed<bf16, float>(p, hd, grid, s);
    case SP_E4M3: return bf16_rows ? read_typed<e4m3, bf16>(p, hd, grid, s) : read_typed<e4m3, float>(p, hd, grid, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace sp
