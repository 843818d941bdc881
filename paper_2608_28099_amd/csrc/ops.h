// Internal interface between the host side of the cache operators (ops.hip) and
// their kernels (cacheops.hip, tree.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sp_probe.h"

namespace sp {

// ---------------------------------------------------------------- rotary
struct RowsArg {
  void* data;
  int64_t row, head;  // strides in elements
};

struct RotaryParams {
  sp_rotary rot;
  const int* positions;
  RowsArg in[2], out[2];  // queries, keys
  int n_heads[2];         // n_heads[1] = 0: no keys
  int n_rows;
  int transpose;
  int vec;                // every head of every array 16-byte aligned
};
// Rows of fp32 (bf16 = 0) or bf16 values.
hipError_t launch_rotary(const RotaryParams& p, int bf16, int n_cus, hipStream_t s);

// ---------------------------------------------------------------- the paged cache
struct StoreArg {
  void *k, *v;
  uint8_t *k_exp, *v_exp;
  int64_t k_sb, k_sh, v_sb, v_sh, e_sb, e_sh;
  int64_t num_blocks;
  const int* block_table;  // nullable (contiguous)
  int bs_log2, mbps, batch, n_kv;
};

struct CacheParams {
  StoreArg st;
  const int *seq_ids, *positions, *src;  // src nullable
  RowsArg k, v;                          // data nullable when reading
  int n_rows, n_src;
  int k_vec, v_vec;                      // heads 16-byte aligned
  int heads_per_wg;
  const sp_rotary* rot;                  // host, nullable (writing)
};
// storage: SP_F32, SP_BF16 or SP_E4M3; bf16: type of the rows.
hipError_t launch_cache_write(const CacheParams& p, int storage, int bf16, int hd, int n_cus, hipStream_t s);
hipError_t launch_cache_read(const CacheParams& p, int storage, int bf16, int hd, hipStream_t s);

// ---------------------------------------------------------------- tree attention
struct TreeParams {
  StoreArg st;
  const int *seq_lens, *counts;  // counts nullable
  const uint32_t* mask;          // nullable: a chain
  int64_t mask_stride;
  int mask_words;
  RowsArg q, k, v, out;
  int q_vec, k_vec, v_vec, o_vec;
  float* lse;                    // nullable
  int nodes, group, max_seq_len;
  float scale_log2;              // the scores' factor times log2(e)
  // the plan: query rows in n_qgroups groups, a workgroup each, of four waves of rows_per_wave (16 or
  // 32) or of eight that share 16 rows (2; fp32 only), r_alloc rows in all; splits of split_len tokens, max_splits of max_seq_len
  int n_qgroups, rows_per_wave, r_alloc, split_len, max_splits;
  float* o_part;                 // [B][n_kv][max_splits][r_alloc / 16][16 hd], not divided by the sum
  float2* ml_part;               // [B][n_kv][max_splits][r_alloc]: maximum (log2 units), sum
};
hipError_t launch_tree(const TreeParams& p, int storage, int hd, hipStream_t s);

}  // namespace sp
