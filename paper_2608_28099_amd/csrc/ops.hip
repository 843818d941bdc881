// Host side of the cache operators (include/sp_probe.h): argument checks, the
// rotation's frequencies and the launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <functional>
#include <mutex>

#include "kernels.h"
#include "ops.h"

#define SP_API extern "C" __attribute__((visibility("default")))

namespace {

using namespace sp;

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool is_pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }
int ilog2(int64_t x) { int r = 0; while ((int64_t(1) << r) < x) ++r; return r; }
int size_of(int dtype) { return dtype == SP_F32 ? 4 : dtype == SP_BF16 ? 2 : 1; }

// Rows of a call.  The cache's kernels take 4 threads per row along the grid's first dimension (less than 2^32 fit); rotations,
// with up to 256 per row, go on along its second.
constexpr int kMaxRows = (1 << 26) - 1;

// The current device: whether the kernels run on it, and its compute units (asked once).
constexpr int kMaxDevices = 64;
struct DeviceInfo {
  std::once_flag once;
  int status, num_cus;
};
DeviceInfo g_devices[kMaxDevices];

void ask_device(DeviceInfo& d, int dev) {
  hipDeviceProp_t prop;
  d.status = SP_ERR_NO_DEVICE;
  if (hipGetDeviceProperties(&prop, dev) != hipSuccess) return;
  if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0) return;
  d.num_cus = prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
  d.status = SP_OK;
}

int current_device(int* num_cus) {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) return SP_ERR_NO_DEVICE;
  if (dev < 0 || dev >= kMaxDevices) return SP_ERR_UNSUPPORTED;
  DeviceInfo& d = g_devices[dev];
  std::call_once(d.once, ask_device, std::ref(d), dev);
  if (d.status == SP_OK) *num_cus = d.num_cus;
  return d.status;
}

int check_rotary(const sp_rotary* r) {
  if (!r || (r->head_dim != 64 && r->head_dim != 128)) return SP_ERR_INVALID_ARG;
  if (r->rotary_dim < 2 || r->rotary_dim > r->head_dim || r->rotary_dim % 2) return SP_ERR_INVALID_ARG;
  if (r->layout != SP_ROTARY_HALF && r->layout != SP_ROTARY_INTERLEAVED) return SP_ERR_INVALID_ARG;
  return SP_OK;
}

// Rows of `heads` heads of esz-byte values; *vec: every head 16-byte aligned.
int check_rows(const sp_rows* r, int heads, int esz, bool* vec) {
  if (!r || !r->data || r->n_heads != heads || r->reserved) return SP_ERR_INVALID_ARG;
  if (!aligned(r->data, esz)) return SP_ERR_INVALID_ARG;
  *vec = *vec && aligned(r->data, 16) && r->stride_row * esz % 16 == 0 && r->stride_head * esz % 16 == 0;
  return SP_OK;
}

RowsArg rows_arg(const sp_rows* r) { return RowsArg{r->data, r->stride_row, r->stride_head}; }

int check_store(const sp_kv_store* s, const int32_t* block_table) {
  if (!s || s->reserved) return SP_ERR_INVALID_ARG;
  if (s->dtype != SP_F32 && s->dtype != SP_BF16 && s->dtype != SP_E4M3) return SP_ERR_INVALID_ARG;
  if (s->head_dim != 64 && s->head_dim != 128) return SP_ERR_UNSUPPORTED;
  if (s->n_kv_heads < 1) return SP_ERR_INVALID_ARG;
  if (s->n_kv_heads > 4096) return SP_ERR_UNSUPPORTED;
  const sp_kv_cache& kv = s->kv;
  if (!kv.k_base || !kv.v_base || !aligned(kv.k_base, 16) || !aligned(kv.v_base, 16)) return SP_ERR_INVALID_ARG;
  if (kv.block_size < 16 || !is_pow2(kv.block_size) || kv.max_blocks_per_seq < 1 || kv.num_blocks < 1 || kv.batch < 0)
    return SP_ERR_INVALID_ARG;
  const int64_t x = 16 / size_of(s->dtype), tile = (int64_t)kv.block_size * s->head_dim;
  if (kv.k_stride_block % x || kv.k_stride_head % x || kv.v_stride_block % x || kv.v_stride_head % x ||
      kv.k_stride_block < 0 || kv.v_stride_block < 0 || kv.k_stride_head < tile || kv.v_stride_head < tile)
    return SP_ERR_INVALID_ARG;
  if (s->dtype == SP_E4M3) {
    if (!s->k_exponents || !s->v_exponents || !aligned(s->k_exponents, 16) || !aligned(s->v_exponents, 16) ||
        s->exponent_stride_block % 16 || s->exponent_stride_head % 16 || s->exponent_stride_block < 0 ||
        s->exponent_stride_head < kv.block_size)
      return SP_ERR_INVALID_ARG;
  }
  if (!block_table && (int64_t)kv.batch * kv.max_blocks_per_seq > kv.num_blocks) return SP_ERR_INVALID_ARG;
  if (block_table && !aligned(block_table, 4)) return SP_ERR_INVALID_ARG;
  return SP_OK;
}

StoreArg store_arg(const sp_kv_store* s, const int32_t* block_table) {
  StoreArg a{};
  a.k = const_cast<void*>(s->kv.k_base);
  a.v = const_cast<void*>(s->kv.v_base);
  a.k_exp = s->k_exponents;
  a.v_exp = s->v_exponents;
  a.k_sb = s->kv.k_stride_block;
  a.k_sh = s->kv.k_stride_head;
  a.v_sb = s->kv.v_stride_block;
  a.v_sh = s->kv.v_stride_head;
  a.e_sb = s->exponent_stride_block;
  a.e_sh = s->exponent_stride_head;
  a.num_blocks = s->kv.num_blocks;
  a.block_table = block_table;
  a.bs_log2 = ilog2(s->kv.block_size);
  a.mbps = s->kv.max_blocks_per_seq;
  a.batch = s->kv.batch;
  a.n_kv = s->n_kv_heads;
  return a;
}

constexpr double kLog2e = 1.4426950408889634;

int check_tree_config(const sp_tree_config* c) {
  if (!c || c->reserved) return SP_ERR_INVALID_ARG;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads) return SP_ERR_INVALID_ARG;
  if (c->dtype != SP_F32 && c->dtype != SP_BF16) return SP_ERR_INVALID_ARG;
  if (c->kv_dtype != SP_F32 && c->kv_dtype != SP_BF16 && c->kv_dtype != SP_E4M3) return SP_ERR_INVALID_ARG;
  if (c->max_nodes < 1 || c->max_batch < 1 || c->max_seq_len < 0) return SP_ERR_INVALID_ARG;
  if (!(c->scale >= 0.f) || !std::isfinite((float)(c->scale * kLog2e))) return SP_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return SP_ERR_UNSUPPORTED;
  if ((c->dtype == SP_F32) != (c->kv_dtype == SP_F32)) return SP_ERR_UNSUPPORTED;
  if (c->max_nodes > 256 || c->n_q_heads > 4096 || c->max_batch > 65535 || c->max_seq_len > 1 << 30) return SP_ERR_UNSUPPORTED;
  return SP_OK;
}

// How a call of `nodes` nodes is laid out on num_cus compute units.  The splits follow the
// config's max_batch, so that its workspace holds every call's partial results.
struct TreePlan {
  int n_qgroups, rows_per_wave, r_alloc, split_len, max_splits;
  size_t part_bytes;  // of O; the (m, l) pairs follow
  size_t total;
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Tokens of a split at least (one sequence of 2048, 240 rows of 8 KV heads, which fill a third of the device: 21.5 us; at
// least 128: 24.3, 192: 23.0, 512: 23.8).
constexpr int kMinSplit = 256;
int64_t slots_of(int num_cus) { return (int64_t)num_cus * 3; }  // three workgroups per compute unit, by LDS

// Rows of a wave, and workgroups that the rows of a KV head take.  Workgroups of four waves, 16 or 32 rows each;
// fp32, while pieces of kMinSplit tokens and 16 rows are two per compute unit at most, of eight waves for 16 rows (2 "rows a
// wave"), which have a shorter way to the first result (8 KV heads, head dim 128, eight waves / four of 16 rows, in us: one
// sequence of 2000 tokens, 4 rows 15.9 / 28.6, 240 rows 59 / 43; 4 of 8000, 4 rows 69 / 53; 48 of 2000, 64 rows
// 566 / 242; 32 of 8000, 240 rows 4110 / 2061).
// A wave of 32 rows reads half as much from LDS per row, but one group of 128 rows in place of two of 64 leaves
// half as many to spread over the device.  So waves of 32 for bf16 caches (whose waves of 16 are bound by LDS) from 129
// rows on, where padding to 128 adds at most a fifth and pieces of kMinSplit tokens would still fill the device
// twice.  The bound on the padding is a compromise: of 160 rows a large call would gain by 32 and a small one lose more.
// Measured (in us, 16 rows a wave / 32): 64 sequences of 6000 tokens: 240 rows 607 / 523, 320 rows 756 / 665,
// 480 rows 1113 / 937; 160 rows, padded to 192 or 256: 487 / 460; 16 of 4000, 160 rows: 76 / 86, 128 rows: 63 / 77;
// 240 rows, 4 of 8000: 56.6 / 55.1, one of 2000: 20.2 / 23.6.  8-bit, when keys were converted to bf16, 64 of 6000: 240
// rows 626 / 652, 320 rows 794 / 873, 480 rows 1189 / 1181; now 577, 727 and 1086 in waves of 16.
void row_groups(const sp_tree_config& c, int nodes, int num_cus, int* rows_per_wave, int* groups) {
  const int rows = nodes * (c.n_q_heads / c.n_kv_heads), g64 = (rows + 63) / 64, g128 = (rows + 127) / 128;
  const bool f32 = c.kv_dtype == SP_F32;
  const int64_t splits = c.max_seq_len < kMinSplit ? 1 : c.max_seq_len / kMinSplit;
  if (f32 && (int64_t)c.max_batch * c.n_kv_heads * ((rows + 15) / 16) * splits <= 2 * num_cus) {
    *rows_per_wave = 2;
    *groups = (rows + 15) / 16;
    return;
  }
  const int64_t pieces = (int64_t)c.max_batch * c.n_kv_heads * g128 * (c.max_seq_len / kMinSplit);
  const bool wide = c.kv_dtype == SP_BF16 && rows > 128 && 5 * 128 * g128 <= 6 * 64 * g64 && pieces >= 2 * slots_of(num_cus);
  *rows_per_wave = wide ? 32 : 16;
  *groups = wide ? g128 : g64;
}

TreePlan tree_plan(const sp_tree_config& c, int nodes, int num_cus) {
  TreePlan p{};
  row_groups(c, nodes, num_cus, &p.rows_per_wave, &p.n_qgroups);
  p.r_alloc = p.n_qgroups * (p.rows_per_wave == 2 ? 16 : 4 * p.rows_per_wave);
  const int64_t items = (int64_t)c.max_batch * c.n_kv_heads * p.n_qgroups;
  const int64_t n = c.max_seq_len, slots = slots_of(num_cus);
  // As many splits as fill the device once, and pieces of at most an eighth of the longest sequence
  // (or 2048 tokens): a batch of long and short sequences takes several rounds, whose ends level
  // out (64 sequences of 2K-32K tokens, 320 rows: 1208 us in the 8 splits of 4096 that this makes of the longest, 1185 in
  // 4, 1279 in 16, 1450 in 32, 1457 unsplit).
  // Then up to as many again, until the last round is full: of alike sequences a round that a third of
  // the device works on costs a whole one (32 of 131072 8-bit tokens, 4 rows: 1414 us in 4 splits
  // each, 1.33 rounds; 1328 in 8, 2.67; 1326 in the 9 that this takes, 3; 1363 in 3, one; 2083 unsplit).
  // The lengths are on the device, so every sequence counts as max_seq_len long here.  Of ragged batches the last round is
  // not where this looks for it: 128 of 1K-8K 8-bit tokens, 64 rows: 215 us in the 5 splits of 1664 that it takes, 198 in
  // 4 of 2048, 224 in 8, 249 unsplit.
  const int64_t fill = (n * items + slots - 1) / slots, cap = n / 8 > 2048 ? n / 8 : 2048;
  int64_t len = fill < cap ? fill : cap;
  if (len < kMinSplit) len = kMinSplit;
  const int64_t k0 = n > len ? (n + len - 1) / len : 1;
  int64_t best = k0;
  double least = 1e30;
  for (int64_t k = k0; k0 > 1 && k <= 2 * k0 && least > 1.1; ++k) {
    const double rounds = (double)(items * k) / (double)slots, waste = std::ceil(rounds) / rounds;
    if (n / k < kMinSplit) break;
    if (waste < least) { least = waste; best = k; }
  }
  len = (n + best - 1) / best;
  if (len < 1) len = 1;
  p.split_len = (int)((len + 63) / 64 * 64);
  p.max_splits = n > 0 ? (int)((n + p.split_len - 1) / p.split_len) : 1;
  if (p.max_splits > 1) {
    const size_t prows = (size_t)c.max_batch * c.n_kv_heads * p.max_splits * p.r_alloc;
    p.part_bytes = align256(prows * c.head_dim * 4);
    p.total = p.part_bytes + align256(prows * 8);
  }
  if (p.total < 256) p.total = 256;
  return p;
}

// The largest plan of the calls that c allows: a plan changes with the groups of rows only.
size_t tree_workspace(const sp_tree_config& c, int num_cus) {
  size_t most = 0;
  int wave0 = 0, groups0 = 0;
  for (int nodes = 1; nodes <= c.max_nodes; ++nodes) {
    int wave, groups;
    row_groups(c, nodes, num_cus, &wave, &groups);
    if (wave == wave0 && groups == groups0) continue;
    wave0 = wave;
    groups0 = groups;
    const size_t x = tree_plan(c, nodes, num_cus).total;
    most = x > most ? x : most;
  }
  return most;
}

}  // namespace

SP_API int sp_probe_rotary_init(const sp_rotary_config* c, sp_rotary* out) {
  if (!c || !out) return SP_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return SP_ERR_UNSUPPORTED;
  if (c->rotary_dim < 2 || c->rotary_dim > c->head_dim || c->rotary_dim % 2) return SP_ERR_INVALID_ARG;
  if (c->layout != SP_ROTARY_HALF && c->layout != SP_ROTARY_INTERLEAVED) return SP_ERR_INVALID_ARG;
  const int dim = c->rotary_dim, half = dim / 2;
  const double two_pi = 6.283185307179586476925;
  auto finite = [](double x) { return std::isfinite(x); };
  double base = c->base, attn = 1.0;
  if (c->scaling != SP_ROTARY_CUSTOM && !(base > 0.0 && finite(base))) return SP_ERR_INVALID_ARG;
  double fast = c->beta_fast, slow = c->beta_slow;
  switch (c->scaling) {
    case SP_ROTARY_PLAIN: break;
    case SP_ROTARY_NTK:
      if (dim == 2) return SP_ERR_INVALID_ARG;  // the exponent has no value
      [[fallthrough]];
    case SP_ROTARY_LINEAR:
      if (!(c->factor >= 1.0 && finite(c->factor))) return SP_ERR_INVALID_ARG;
      if (c->scaling == SP_ROTARY_NTK) base *= std::pow(c->factor, dim / (dim - 2.0));
      break;
    case SP_ROTARY_YARN:
      if (!(c->factor >= 1.0 && finite(c->factor))) return SP_ERR_INVALID_ARG;
      if (!(c->original_positions > 0.0 && finite(c->original_positions))) return SP_ERR_INVALID_ARG;
      if (fast == 0.0 && slow == 0.0) { fast = 32.0; slow = 1.0; }
      if (!(slow >= 0.0 && fast > slow && finite(fast))) return SP_ERR_INVALID_ARG;
      if (!(c->attn_factor >= 0.0 && finite(c->attn_factor))) return SP_ERR_INVALID_ARG;
      attn = c->attn_factor > 0.0 ? c->attn_factor : 0.1 * std::log(c->factor) + 1.0;
      break;
    case SP_ROTARY_CUSTOM:
      if (!c->frequencies || !(c->attn_factor >= 0.0 && finite(c->attn_factor))) return SP_ERR_INVALID_ARG;
      attn = c->attn_factor > 0.0 ? c->attn_factor : 1.0;
      break;
    default: return SP_ERR_INVALID_ARG;
  }
  sp_rotary r{};
  r.head_dim = c->head_dim;
  r.rotary_dim = dim;
  r.layout = c->layout;
  r.scale = (float)attn;
  if (!std::isfinite(r.scale)) return SP_ERR_INVALID_ARG;
  for (int p = 0; p < half; ++p) {
    double theta = c->scaling == SP_ROTARY_CUSTOM ? c->frequencies[p] : std::pow(base, -2.0 * p / dim);
    if (c->scaling == SP_ROTARY_LINEAR) theta /= c->factor;
    if (c->scaling == SP_ROTARY_YARN) {
      double g = (c->original_positions * theta / two_pi - slow) / (fast - slow);
      g = g < 0.0 ? 0.0 : (g > 1.0 ? 1.0 : g);
      theta = (1.0 - g) * theta / c->factor + g * theta;
    }
    r.turns[p] = theta / two_pi;
    // whole turns of any position are counted in 64 bits (bases below 1 make theta grow)
    if (!(std::fabs(r.turns[p]) <= 1.0e9)) return SP_ERR_INVALID_ARG;
  }
  *out = r;
  return SP_OK;
}

SP_API int sp_probe_rotary(const sp_rotary* rot, int32_t dtype, int32_t transpose, int32_t n_rows,
                           const int32_t* positions, const sp_rows* q, const sp_rows* q_out, const sp_rows* k,
                           const sp_rows* k_out, void* stream) {
  int st = check_rotary(rot);
  if (st != SP_OK) return st;
  if (dtype != SP_F32 && dtype != SP_BF16) return SP_ERR_INVALID_ARG;
  if (n_rows < 0 || !q || !q_out || (k == nullptr) != (k_out == nullptr)) return SP_ERR_INVALID_ARG;
  if (q->n_heads < 1 || (k && k->n_heads < 1)) return SP_ERR_INVALID_ARG;
  if (q->n_heads > 4096 || (k && k->n_heads > 4096)) return SP_ERR_UNSUPPORTED;
  if (n_rows > kMaxRows) return SP_ERR_UNSUPPORTED;
  if (n_rows == 0) return SP_OK;
  if (!positions || !aligned(positions, 4)) return SP_ERR_INVALID_ARG;
  const int esz = size_of(dtype);
  bool vec = true;
  RotaryParams p{};
  const sp_rows* in[2] = {q, k};
  const sp_rows* out[2] = {q_out, k_out};
  for (int a = 0; a < (k ? 2 : 1); ++a) {
    if ((st = check_rows(in[a], in[a]->n_heads, esz, &vec)) != SP_OK) return st;
    if ((st = check_rows(out[a], in[a]->n_heads, esz, &vec)) != SP_OK) return st;
    p.in[a] = rows_arg(in[a]);
    p.out[a] = rows_arg(out[a]);
    p.n_heads[a] = in[a]->n_heads;
  }
  int cus = 0;
  if ((st = current_device(&cus)) != SP_OK) return st;
  p.rot = *rot;
  p.positions = positions;
  p.n_rows = n_rows;
  p.transpose = transpose != 0;
  p.vec = vec;
  return launch_rotary(p, dtype == SP_BF16, cus, (hipStream_t)stream) == hipSuccess ? SP_OK : SP_ERR_HIP;
}

namespace {

// The checks and parameters that writing and reading share.
int cache_params(const sp_kv_store* store, const int32_t* block_table, int32_t dtype, int32_t n_rows,
                 const int32_t* seq_ids, const int32_t* positions, const sp_rows* k, const sp_rows* v,
                 CacheParams* p) {
  int st = check_store(store, block_table);
  if (st != SP_OK) return st;
  if (dtype != SP_F32 && dtype != SP_BF16) return SP_ERR_INVALID_ARG;
  if (n_rows < 0) return SP_ERR_INVALID_ARG;
  if (n_rows > kMaxRows) return SP_ERR_UNSUPPORTED;
  if (n_rows == 0) return SP_OK;
  if (!seq_ids || !positions || !aligned(seq_ids, 4) || !aligned(positions, 4)) return SP_ERR_INVALID_ARG;
  bool k_vec = true, v_vec = true;
  if (k) {
    if ((st = check_rows(k, store->n_kv_heads, size_of(dtype), &k_vec)) != SP_OK) return st;
    p->k = rows_arg(k);
  }
  if (v) {
    if ((st = check_rows(v, store->n_kv_heads, size_of(dtype), &v_vec)) != SP_OK) return st;
    p->v = rows_arg(v);
  }
  p->k_vec = k_vec;
  p->v_vec = v_vec;
  p->st = store_arg(store, block_table);
  p->seq_ids = seq_ids;
  p->positions = positions;
  p->n_rows = n_rows;
  return SP_OK;
}

}  // namespace

SP_API int sp_probe_cache_write(const sp_kv_store* store, const int32_t* block_table, int32_t dtype, int32_t n_rows,
                                const int32_t* seq_ids, const int32_t* positions, const int32_t* src_rows,
                                int32_t n_src, const sp_rows* k, const sp_rows* v, const sp_rotary* rot,
                                void* stream) {
  CacheParams p{};
  // no source row: every row is skipped, k and v need not exist
  const bool none = n_src == 0;
  int st = cache_params(store, block_table, dtype, n_rows, seq_ids, positions, none ? nullptr : k, none ? nullptr : v, &p);
  if (st != SP_OK) return st;
  if (rot) {
    if ((st = check_rotary(rot)) != SP_OK) return st;
    if (rot->head_dim != store->head_dim) return SP_ERR_INVALID_ARG;
  }
  if (n_src < 0) return SP_ERR_INVALID_ARG;
  if (n_rows == 0 || none) return SP_OK;
  if (!k || !v || (src_rows && !aligned(src_rows, 4))) return SP_ERR_INVALID_ARG;
  int cus = 0;
  if ((st = current_device(&cus)) != SP_OK) return st;
  p.src = src_rows;
  p.n_src = n_src;
  p.rot = rot;
  return launch_cache_write(p, store->dtype, dtype == SP_BF16, store->head_dim, cus, (hipStream_t)stream) == hipSuccess
             ? SP_OK : SP_ERR_HIP;
}

SP_API int sp_probe_cache_read(const sp_kv_store* store, const int32_t* block_table, int32_t dtype, int32_t n_rows,
                               const int32_t* seq_ids, const int32_t* positions, const sp_rows* k, const sp_rows* v,
                               void* stream) {
  CacheParams p{};
  int st = cache_params(store, block_table, dtype, n_rows, seq_ids, positions, k, v, &p);
  if (st != SP_OK) return st;
  if (n_rows == 0 || (!k && !v)) return SP_OK;
  int cus = 0;
  if ((st = current_device(&cus)) != SP_OK) return st;
  p.n_src = n_rows;
  return launch_cache_read(p, store->dtype, dtype == SP_BF16, store->head_dim, (hipStream_t)stream) == hipSuccess
             ? SP_OK : SP_ERR_HIP;
}

SP_API size_t sp_probe_tree_workspace_bytes(const sp_tree_config* cfg) {
  if (check_tree_config(cfg) != SP_OK) return 0;
  int cus = 256;
  if (current_device(&cus) != SP_OK) cus = 256;
  return tree_workspace(*cfg, cus);
}

SP_API int sp_probe_tree_attention(const sp_tree_config* c, const sp_kv_store* store, const int32_t* seq_lens,
                                   const int32_t* block_table, const sp_tree* t, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  int st = check_tree_config(c);
  if (st != SP_OK) return st;
  if ((st = check_store(store, block_table)) != SP_OK) return st;
  if (!t) return SP_ERR_INVALID_ARG;
  if (store->dtype != c->kv_dtype || store->n_kv_heads != c->n_kv_heads || store->head_dim != c->head_dim)
    return SP_ERR_INVALID_ARG;
  if ((int64_t)store->kv.max_blocks_per_seq * store->kv.block_size < (int64_t)c->max_seq_len) return SP_ERR_INVALID_ARG;
  // places within a head's block are 32-bit byte offsets in the kernels (signed ones on the way)
  if ((int64_t)store->kv.block_size * c->head_dim * size_of(c->kv_dtype) > (int64_t)1 << 31) return SP_ERR_UNSUPPORTED;
  if (t->n_nodes < 1) return SP_ERR_INVALID_ARG;
  if (t->n_nodes > c->max_nodes || store->kv.batch > c->max_batch) return SP_ERR_CAPACITY;
  if (t->mask && (t->mask_words < (t->n_nodes + 31) / 32 || t->mask_stride < 0 || !aligned(t->mask, 4)))
    return SP_ERR_INVALID_ARG;
  if (store->kv.batch == 0) return SP_OK;
  if (!seq_lens || !aligned(seq_lens, 4) || !aligned(t->counts, 4) || !aligned(t->lse, 4)) return SP_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 16)) return SP_ERR_INVALID_ARG;
  TreeParams p{};
  const int esz = size_of(c->dtype);
  bool q_vec = true, k_vec = true, v_vec = true, o_vec = true;
  if ((st = check_rows(&t->q, c->n_q_heads, esz, &q_vec)) != SP_OK) return st;
  if ((st = check_rows(&t->k, c->n_kv_heads, esz, &k_vec)) != SP_OK) return st;
  if ((st = check_rows(&t->v, c->n_kv_heads, esz, &v_vec)) != SP_OK) return st;
  if ((st = check_rows(&t->out, c->n_q_heads, esz, &o_vec)) != SP_OK) return st;
  int cus = 0;
  st = current_device(&cus);
  const TreePlan pl = tree_plan(*c, t->n_nodes, st == SP_OK ? cus : 256);
  if (workspace_bytes < pl.total) return SP_ERR_INVALID_ARG;
  if (st != SP_OK) return st;
  p.n_qgroups = pl.n_qgroups;
  p.rows_per_wave = pl.rows_per_wave;
  p.r_alloc = pl.r_alloc;
  p.split_len = pl.split_len;
  p.max_splits = pl.max_splits;
  p.o_part = (float*)workspace;
  p.ml_part = (float2*)((char*)workspace + pl.part_bytes);
  p.st = store_arg(store, block_table);
  p.seq_lens = seq_lens;
  p.counts = t->counts;
  p.mask = t->mask;
  p.mask_stride = t->mask_stride;
  p.mask_words = t->mask_words;
  p.q = rows_arg(&t->q);
  p.k = rows_arg(&t->k);
  p.v = rows_arg(&t->v);
  p.out = rows_arg(&t->out);
  p.q_vec = q_vec;
  p.k_vec = k_vec;
  p.v_vec = v_vec;
  p.o_vec = o_vec;
  p.lse = t->lse;
  p.nodes = t->n_nodes;
  p.group = c->n_q_heads / c->n_kv_heads;
  p.max_seq_len = c->max_seq_len;
  const double scale = c->scale > 0.f ? (double)c->scale : 1.0 / std::sqrt((double)c->head_dim);
  p.scale_log2 = (float)(scale * kLog2e);
  return launch_tree(p, c->kv_dtype, c->head_dim, (hipStream_t)stream) == hipSuccess ? SP_OK : SP_ERR_HIP;
}
