// C ABI of the operators around a key/value cache held in 4 bits (see include/headcast.h): rotary positions, packing, attention,
// accumulated attention weights and eviction.  Nothing here allocates device memory, copies to the host or waits, except
// headcast_packed_check; a cache's memory and every workspace are the caller's.
#include "../../include/headcast.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <type_traits>

#include "evict_kernels.cuh"
#include "launch.h"
#include "packed_attn_kernel.cuh"
#include "packed_kernels.cuh"
#include "packed_observe_kernel.cuh"
#include "packed_rows_kernel.cuh"
#include "rope_kernel.cuh"
#include "tmap.h"
#include "turns.h"

using namespace hc;

struct headcast_packed {
  headcast_packed_config cfg;
  PackedView view;
  int64_t bytes = 0;  // of the storage, from view.status on
  int device = 0, n_sm = 0;
  float scale = 0.f;
  int32_t len[PACK_MAX_HEADS] = {};
  unsigned configured = 0;  // kernels whose dynamic shared memory has been set, a bit each
  char error[256] = "";
};

namespace {

int fail(headcast_packed* c, int code, const char* fmt, ...) {
  va_list args;
  va_start(args, fmt);
  vsnprintf(c->error, sizeof(c->error), fmt, args);
  va_end(args);
  return code;
}
#define PK_CUDA(c, call)                                                                                          \
  do {                                                                                                            \
    const cudaError_t e_ = (call);                                                                                \
    if (e_ != cudaSuccess) {                                                                                      \
      cudaGetLastError(); /* reported here, and by no later call */                                               \
      return fail(c, e_ == cudaErrorMemoryAllocation ? HC_ERR_NOMEM : HC_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_)); \
    }                                                                                                             \
  } while (0)

bool aligned(const void* p, uintptr_t to = 16) { return p && reinterpret_cast<uintptr_t>(p) % to == 0; }

// [a, a + bytes_a) and [b, b + bytes_b) share a byte
bool overlap(const void* a, int64_t bytes_a, const void* b, int64_t bytes_b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + static_cast<uintptr_t>(bytes_b) && y < x + static_cast<uintptr_t>(bytes_a);
}

int64_t round_up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

bool config_ok(const headcast_packed_config* cfg) {
  return cfg && cfg->n_heads >= 1 && cfg->n_heads <= PACK_MAX_HEADS && cfg->n_kv_heads >= 1 && cfg->n_heads % cfg->n_kv_heads == 0 &&
         (cfg->head_dim == 64 || cfg->head_dim == 128) && cfg->capacity >= 1 && cfg->capacity <= HEADCAST_PACKED_MAX_TOKENS &&
         (cfg->softmax_scale == 0.f || (cfg->softmax_scale >= 0x1p-40f && cfg->softmax_scale <= 0x1p40f));
}

// Offsets of the planes in the storage; returns its size.
int64_t layout(const headcast_packed_config& cfg, int64_t (&at)[5]) {
  const int64_t rows = round_up(cfg.capacity, PACK_TILE) * cfg.n_kv_heads;
  const int64_t sizes[5] = {rows * cfg.head_dim / 2, rows * cfg.head_dim / 2, rows * cfg.head_dim / PACK_GROUP, rows * cfg.head_dim / PACK_GROUP, rows * 4};
  int64_t total = 256;  // the status word
  for (int i = 0; i < 5; ++i) {
    at[i] = total;
    total += round_up(sizes[i], 256);
  }
  return total;
}

bool in_storage(const headcast_packed* c, const void* p, int64_t bytes) { return overlap(c->view.status, c->bytes, p, bytes); }

// A call's cache and device: HC_OK, or the reason in the cache.
int enter(headcast_packed* c) {
  if (!c) return HC_ERR_INVALID_ARG;
  int dev = -1;
  PK_CUDA(c, cudaGetDevice(&dev));
  if (dev != c->device) return fail(c, HC_ERR_INVALID_ARG, "the cache lives on device %d, the current device is %d", c->device, dev);
  return HC_OK;
}

// The attribute belongs to the function in a CUDA context: every cache sets it once for itself, whatever GPU it is on.
enum { KERNEL_ROWS = 1, KERNEL_ATTN = 2, KERNEL_OBSERVE = 4, KERNEL_ROWS_16 = 8 };
template <typename K>
int allow_smem(headcast_packed* c, unsigned which, K* kernel, int bytes) {
  if (c->configured & which) return HC_OK;
  PK_CUDA(c, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  c->configured |= which;
  return HC_OK;
}

HeadCounts lengths(const headcast_packed* c) {
  HeadCounts n;
  std::memset(&n, 0, sizeof(n));
  for (int h = 0; h < c->cfg.n_kv_heads; ++h) n.n[h] = c->len[h];
  return n;
}
// first[h]: steps of the heads before h, per_tile for each of their tiles.  Returns the steps of all.
template <typename T>
T step_line(const headcast_packed* c, T (&first)[PACK_MAX_HEADS + 1], T per_tile) {
  T total = 0;
  for (int h = 0; h <= PACK_MAX_HEADS; ++h) {
    first[h] = total;
    if (h < c->cfg.n_kv_heads) total += (c->len[h] + PACK_TILE - 1) / PACK_TILE * per_tile;
  }
  return total;
}

// Up to 16 rows per key/value head go to packed_rows_kernel: 16 x 32760 tokens, 12 heads of 128, 27 us; packed_attn_kernel, for which
// 17 rows are as much work as 128, takes 48.  Observing, packed_observe_rows_kernel takes 11.8 us for 16 rows (9.1 for one), and
// packed_observe_kernel 32 for 17.
bool few_rows(const headcast_packed* c, int32_t n_queries) { return static_cast<int64_t>(n_queries) * (c->cfg.n_heads / c->cfg.n_kv_heads) <= ROWS_MAX; }

struct RowsWorkspace {
  int64_t part_o, part_ml, bytes;
  explicit RowsWorkspace(const headcast_packed* c) {
    const int64_t slots = c->n_sm + c->cfg.n_kv_heads;
    part_o = 0;
    part_ml = slots * ROWS_MAX * c->cfg.head_dim * 4;
    bytes = part_ml + slots * ROWS_MAX * 8;
  }
};

template <int D>
int attend_few(headcast_packed* c, const void* q, void* out, float* lse, int32_t n_queries, void* ws, cudaStream_t st) {
  const RowsWorkspace w(c);
  PackedRowsParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = c->view;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.part_o);
  p.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + w.part_ml);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.n_queries = n_queries;
  p.group = c->cfg.n_heads / c->cfg.n_kv_heads;
  p.n_rows = n_queries * p.group;
  p.scale_log2e = c->scale * 1.4426950408889634f;
  p.len = lengths(c);
  const int total = step_line(c, p.tile_first, 1);
  p.n_cta = std::min(c->n_sm, total);
  if (total > 0) {
    const bool one = p.n_rows <= 8;  // 32760 tokens, 12 heads of 128: 18.1 us; with two tiles of queries 26.7
    const int smem = RowsSmem<D>::DYN_BYTES;
    auto* kernel = one ? packed_rows_kernel<D, 1> : packed_rows_kernel<D, 2>;
    const int rc = allow_smem(c, one ? KERNEL_ROWS : KERNEL_ROWS_16, kernel, smem);
    if (rc != HC_OK) return rc;
    PK_CUDA(c, launch_pdl(kernel, dim3(p.n_cta), dim3(ROWS_THREADS), smem, st, p));
  }
  PK_CUDA(c, launch_pdl(packed_merge_rows_kernel<D>, dim3(p.n_rows, c->cfg.n_kv_heads), dim3(MERGE_GROUPS * D / 4), 0, st, p));
  return HC_OK;
}

struct ManyWorkspace {
  int64_t part_o, part_ml, bytes;
  explicit ManyWorkspace(const headcast_packed* c) {
    const int64_t rows = 2ll * c->n_sm * 256;
    part_o = 0;
    part_ml = rows * c->cfg.head_dim * 4;
    bytes = part_ml + rows * 8;
  }
};

template <int D>
int attend_many(headcast_packed* c, const void* q, void* out, float* lse, int32_t n_queries, void* ws, cudaStream_t st) {
  const ManyWorkspace w(c);
  PackedAttnParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = c->view;
  p.q = static_cast<const __nv_bfloat16*>(q);
  p.out = static_cast<__nv_bfloat16*>(out);
  p.lse = lse;
  p.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + w.part_o);
  p.part_ml = reinterpret_cast<float2*>(static_cast<uint8_t*>(ws) + w.part_ml);
  p.n_queries = n_queries;
  p.group = c->cfg.n_heads / c->cfg.n_kv_heads;
  p.n_rows = n_queries * p.group;
  p.n_pairs = (p.n_rows + 255) / 256;
  p.scale_log2e = c->scale * 1.4426950408889634f;
  p.len = lengths(c);
  const int64_t total = step_line<int64_t>(c, p.line_first, p.n_pairs);
  p.n_cta = static_cast<int32_t>(std::min<int64_t>(c->n_sm, total));
  bool empty = false;
  int64_t parts = 0;  // of a pair, at most
  for (int h = 0; h < c->cfg.n_kv_heads; ++h) {
    const int64_t tiles = (c->len[h] + PACK_TILE - 1) / PACK_TILE;
    empty = empty || tiles == 0;
    if (total > 0) parts = std::max(parts, tiles * p.n_cta / total + 2);
  }
  if (total > 0) {
    const int rc = allow_smem(c, KERNEL_ATTN, packed_attn_kernel<D>, PackedAttnSmem<D>::DYN_BYTES);
    if (rc != HC_OK) return rc;
    PK_CUDA(c, launch_pdl(packed_attn_kernel<D>, dim3(p.n_cta), dim3(PATTN_THREADS), PackedAttnSmem<D>::DYN_BYTES, st, p));
    if (p.n_cta > 1) {
      int64_t pairs = 0;
      for (int h = 0; h < c->cfg.n_kv_heads; ++h) pairs += c->len[h] > 0 ? p.n_pairs : 0;
      const bool by_pair = pairs < p.n_cta - 1;
      // Groups of threads that share a row's parts: with one 57 us for 700 queries x 9000 tokens (6 parts a pair; with four 65, with sixteen
      // 94), with four 23.8 us for 77 x 10007, 16 / 4 heads of 64 (20 parts; 26.5 and 25.4), with sixteen 23 us for 200 x 25000, one head
      // (148 parts; 78 and 36).
      const int groups = parts <= 10 ? 1 : parts <= 24 ? 4 : 16;
      auto* merge = groups == 1 ? packed_merge_kernel<D, 1> : groups == 4 ? packed_merge_kernel<D, 4> : packed_merge_kernel<D, 16>;
      PK_CUDA(c, launch_pdl(merge, dim3((by_pair ? static_cast<int>(pairs) : p.n_cta - 1) * 16 * groups), dim3(16 * D / 8), 0, st, p, by_pair));
    }
  }
  if (empty) {
    const int rows = 256 / (D / 8);
    PK_CUDA(c, launch_pdl(packed_empty_kernel<D>, dim3((p.n_rows + rows - 1) / rows, c->cfg.n_kv_heads), dim3(256), 0, st, p));
  }
  return HC_OK;
}

thread_local char g_rope_error[256] = "";

int rope_fail(int code, const char* msg) {
  snprintf(g_rope_error, sizeof(g_rope_error), "%s", msg);
  return code;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------------------------- rotary positions

void headcast_rope_default_config(headcast_rope_config* cfg) {
  if (!cfg) return;
  std::memset(cfg, 0, sizeof(*cfg));
  cfg->theta = 10000.0;
  cfg->scale_t = cfg->scale_h = cfg->scale_w = 1.0;
}

const char* headcast_rope_last_error(void) { return g_rope_error; }

int headcast_rope(const headcast_rope_config* cfg, const void* q, void* q_out, int64_t q_stride, const void* k, void* k_out, int64_t k_stride,
                  int32_t n_tokens, int64_t first_frame, const int32_t* positions, int32_t inverse, void* stream) {
  if (!cfg) return rope_fail(HC_ERR_INVALID_ARG, "null config");
  const int64_t d = cfg->head_dim, width = static_cast<int64_t>(cfg->dim_t) + cfg->dim_h + cfg->dim_w;
  if ((d != 64 && d != 128) || cfg->n_heads < 1 || cfg->n_heads > PACK_MAX_HEADS || cfg->n_kv_heads < 0 || cfg->n_kv_heads > PACK_MAX_HEADS)
    return rope_fail(HC_ERR_INVALID_ARG, "sizes out of range (head_dim 64 or 128, 1..64 heads)");
  if (cfg->dim_t < 0 || cfg->dim_h < 0 || cfg->dim_w < 0 || ((cfg->dim_t | cfg->dim_h | cfg->dim_w) & 1) || width < 2 || width > d)
    return rope_fail(HC_ERR_INVALID_ARG, "the axes' widths must be even, not negative, and between 2 and head_dim together");
  if (cfg->halves && width % 16 != 0) return rope_fail(HC_ERR_UNSUPPORTED, "halves need a rotated width that is a multiple of 16");
  if (!(cfg->theta > 0.0 && std::isfinite(cfg->theta)) || !std::isfinite(cfg->scale_t) || !std::isfinite(cfg->scale_h) || !std::isfinite(cfg->scale_w))
    return rope_fail(HC_ERR_INVALID_ARG, "theta must be positive, theta and the scales finite");
  if (n_tokens > 0 && !positions && (cfg->grid_h < 1 || cfg->grid_w < 1 || static_cast<int64_t>(cfg->grid_h) * cfg->grid_w > INT32_MAX))
    return rope_fail(HC_ERR_INVALID_ARG, "without positions the grid must be given");
  if (n_tokens < 0) return rope_fail(HC_ERR_INVALID_ARG, "n_tokens must not be negative");
  if (first_frame < -(int64_t(1) << 31) || first_frame > (int64_t(1) << 31)) return rope_fail(HC_ERR_INVALID_ARG, "first_frame out of range");
  if ((k == nullptr) != (k_out == nullptr) || (k && cfg->n_kv_heads < 1)) return rope_fail(HC_ERR_INVALID_ARG, "k, k_out and n_kv_heads belong together");
  if (positions && !aligned(positions, 4)) return rope_fail(HC_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  if (n_tokens == 0) return HC_OK;
  RopeParams p;
  std::memset(&p, 0, sizeof(p));
  const void* src[2] = {q, k};
  void* dst[2] = {q_out, k_out};
  const int64_t strides[2] = {q_stride, k_stride};
  const int heads[2] = {cfg->n_heads, cfg->n_kv_heads};
  int64_t src_bytes[2] = {0, 0}, dst_bytes[2] = {0, 0};
  for (int i = 0; i < (k ? 2 : 1); ++i) {
    const int64_t row = heads[i] * d, stride = strides[i] ? strides[i] : row;
    if (!aligned(src[i]) || !aligned(dst[i])) return rope_fail(HC_ERR_INVALID_ARG, "q, k and their outputs must be 16-byte aligned device pointers");
    if (stride < row || stride % 8 != 0 || stride >= (int64_t(1) << 31)) return rope_fail(HC_ERR_INVALID_ARG, "a token stride must cover the token's heads and be a multiple of 8 elements");
    src_bytes[i] = 2 * (stride * (n_tokens - 1) + row);
    dst_bytes[i] = 2 * row * n_tokens;
    p.src[i] = static_cast<const __nv_bfloat16*>(src[i]);
    p.dst[i] = static_cast<__nv_bfloat16*>(dst[i]);
    p.src_stride[i] = stride;
    p.heads[i] = heads[i];
  }
  // an output may be its own source; anything else that overlaps would be read after it was written
  for (int i = 0; i < (k ? 2 : 1); ++i)
    for (int j = 0; j < (k ? 2 : 1); ++j) {
      const bool same = i == j && src[i] == dst[i] && p.src_stride[i] == heads[i] * d;
      if (!same && overlap(src[i], src_bytes[i], dst[j], dst_bytes[j])) return rope_fail(HC_ERR_INVALID_ARG, "an output overlaps an input that it is not");
      if (i == j && positions && overlap(positions, 12ll * n_tokens, dst[i], dst_bytes[i])) return rope_fail(HC_ERR_INVALID_ARG, "an output overlaps the positions");
      if (i < j && overlap(dst[i], dst_bytes[i], dst[j], dst_bytes[j])) return rope_fail(HC_ERR_INVALID_ARG, "the outputs overlap");
    }
  p.n = n_tokens;
  p.pairs = static_cast<int32_t>(width / 2);
  p.pairs_t = cfg->dim_t / 2;
  p.pairs_th = (cfg->dim_t + cfg->dim_h) / 2;
  p.grid_w = positions ? 1 : cfg->grid_w;
  p.frame_tokens = positions ? 1 : cfg->grid_h * cfg->grid_w;
  p.first_frame = first_frame;
  p.positions = positions;
  const int dims[3] = {cfg->dim_t, cfg->dim_h, cfg->dim_w};
  const double scales[3] = {cfg->scale_t, cfg->scale_h, cfg->scale_w};
  for (int a = 0, i = 0; a < 3; ++a) {
    // One root per axis; the j-th product is off by (2 + 4 j) 2^-64 of itself.
    const Extended ratio = dims[a] > 2 ? inverse_root(cfg->theta, dims[a] / 2) : Extended{};
    Extended turns = product(extended(std::fabs(scales[a])), TURNS_PER_RADIAN);
    for (int j = 0; j < dims[a] / 2; ++j, ++i, turns = product(turns, ratio)) {
      if (turns.e > 1024) return rope_fail(HC_ERR_INVALID_ARG, "a frequency is not finite");
      const uint64_t f = fraction_of_turn(turns);  // whole turns per position change nothing
      p.frequency[i] = (scales[a] < 0.0) != (inverse != 0) ? 0 - f : f;
    }
  }
  // Tokens of a block (their sines and cosines are formed once for all heads): 4 where every SM gets a few blocks (three frames of 45 x 80,
  // pairs side by side, 27.8 us and of 68 x 120 56.6; 8 tokens 32.3 and 58.1, 16 tokens 37.6 and 67), fewer in small calls.
  int per_block = 4;
  while (per_block > 1 && (n_tokens + per_block - 1) / per_block < ROPE_MANY_BLOCKS) per_block /= 2;
  const dim3 grid((n_tokens + per_block - 1) / per_block);
  const size_t smem = static_cast<size_t>(per_block) * (d / 2) * sizeof(float2);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto* kernel = d == 128 ? (cfg->halves ? rope_kernel<128, true> : rope_kernel<128, false>) : (cfg->halves ? rope_kernel<64, true> : rope_kernel<64, false>);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(ROPE_THREADS), smem, st, p, per_block);
  if (e != cudaSuccess) {
    cudaGetLastError();
    return rope_fail(HC_ERR_CUDA, cudaGetErrorString(e));
  }
  return HC_OK;
}

// ---------------------------------------------------------------------------------------------- the packed cache

int64_t headcast_packed_bytes(const headcast_packed_config* cfg) {
  if (!config_ok(cfg)) return HC_ERR_INVALID_ARG;
  int64_t at[5];
  return layout(*cfg, at);
}

int headcast_packed_create(const headcast_packed_config* cfg, void* storage, int64_t storage_bytes, void* stream, headcast_packed** out) {
  if (!out) return HC_ERR_INVALID_ARG;
  *out = nullptr;
  if (!config_ok(cfg) || !aligned(storage, 256)) return HC_ERR_INVALID_ARG;
  int64_t at[5];
  if (storage_bytes < layout(*cfg, at)) return HC_ERR_INVALID_ARG;
  headcast_packed* c = new (std::nothrow) headcast_packed();
  if (!c) return HC_ERR_NOMEM;
  int major = 0;
  int rc = HC_OK;
  if (cudaGetDevice(&c->device) != cudaSuccess || cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, c->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&c->n_sm, cudaDevAttrMultiProcessorCount, c->device) != cudaSuccess)
    rc = HC_ERR_CUDA;
  else if (major != 10)
    rc = HC_ERR_UNSUPPORTED;
  else if (cudaMemsetAsync(storage, 0, sizeof(int32_t), static_cast<cudaStream_t>(stream)) != cudaSuccess)
    rc = HC_ERR_CUDA;
  if (rc != HC_OK) {
    cudaGetLastError();
    delete c;
    return rc;
  }
  c->cfg = *cfg;
  c->bytes = layout(*cfg, at);
  c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt(static_cast<float>(cfg->head_dim));
  uint8_t* base = static_cast<uint8_t*>(storage);
  c->view.status = reinterpret_cast<int32_t*>(base);
  c->view.k_codes = base + at[0];
  c->view.v_codes = base + at[1];
  c->view.k_scales = base + at[2];
  c->view.v_scales = base + at[3];
  c->view.weights = reinterpret_cast<float*>(base + at[4]);
  c->view.cap = round_up(cfg->capacity, PACK_TILE);
  c->view.n_kv = cfg->n_kv_heads;
  c->view.head_dim = cfg->head_dim;
  *out = c;
  return HC_OK;
}

int headcast_packed_destroy(headcast_packed* c) {
  delete c;
  return HC_OK;
}

const char* headcast_packed_last_error(const headcast_packed* c) { return c ? c->error : "null cache"; }

int headcast_packed_lengths(const headcast_packed* c, int32_t* lengths_host) {
  if (!c || !lengths_host) return HC_ERR_INVALID_ARG;
  std::memcpy(lengths_host, c->len, c->cfg.n_kv_heads * sizeof(int32_t));
  return HC_OK;
}

int headcast_packed_clear(headcast_packed* c) {
  if (!c) return HC_ERR_INVALID_ARG;
  std::memset(c->len, 0, sizeof(c->len));
  return HC_OK;
}

int headcast_packed_drop_last(headcast_packed* c, int32_t n_tokens) {
  if (!c) return HC_ERR_INVALID_ARG;
  if (n_tokens < 0) return fail(c, HC_ERR_INVALID_ARG, "n_tokens must not be negative");
  for (int h = 0; h < c->cfg.n_kv_heads; ++h)
    if (c->len[h] < n_tokens) return fail(c, HC_ERR_STATE, "head %d holds %d tokens, %d were to go", h, c->len[h], n_tokens);
  for (int h = 0; h < c->cfg.n_kv_heads; ++h) c->len[h] -= n_tokens;
  return HC_OK;
}

int64_t headcast_packed_weights_offset(const headcast_packed* c, int64_t* row_stride) {
  if (!c) return HC_ERR_INVALID_ARG;
  if (row_stride) *row_stride = c->view.cap;
  return reinterpret_cast<uint8_t*>(c->view.weights) - reinterpret_cast<uint8_t*>(c->view.status);
}

int headcast_packed_append(headcast_packed* c, const void* k, const void* v, int32_t n_tokens, int64_t token_stride, void* stream) {
  const int rc = enter(c);
  if (rc != HC_OK) return rc;
  if (n_tokens < 0) return fail(c, HC_ERR_INVALID_ARG, "n_tokens must not be negative");
  if (n_tokens == 0) return HC_OK;
  const int64_t row = static_cast<int64_t>(c->cfg.n_kv_heads) * c->cfg.head_dim, stride = token_stride ? token_stride : row;
  if (!aligned(k) || !aligned(v)) return fail(c, HC_ERR_INVALID_ARG, "k and v must be 16-byte aligned device pointers");
  if (stride < row || stride % 8 != 0 || stride >= (int64_t(1) << 31))
    return fail(c, HC_ERR_INVALID_ARG, "a token stride must cover the token's heads and be a multiple of 8 elements");
  for (int h = 0; h < c->cfg.n_kv_heads; ++h)
    if (n_tokens > c->cfg.capacity - c->len[h])
      return fail(c, HC_ERR_STATE, "head %d holds %d tokens of at most %d: no room for %d more", h, c->len[h], c->cfg.capacity, n_tokens);
  const int64_t bytes = 2 * (stride * (n_tokens - 1) + row);
  if (in_storage(c, k, bytes) || in_storage(c, v, bytes)) return fail(c, HC_ERR_INVALID_ARG, "k or v overlaps the cache's storage");
  PackParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = c->view;
  p.k = static_cast<const __nv_bfloat16*>(k);
  p.v = static_cast<const __nv_bfloat16*>(v);
  p.stride = stride;
  p.n = n_tokens;
  p.first = lengths(c);
  const int rows = pack_block_tokens(c->cfg.head_dim);
  PK_CUDA(c, launch_pdl(c->cfg.head_dim == 128 ? pack_rows_kernel<128> : pack_rows_kernel<64>, dim3((n_tokens + rows - 1) / rows, c->cfg.n_kv_heads, 2),
                        dim3(PACK_THREADS), 0, static_cast<cudaStream_t>(stream), p));
  for (int h = 0; h < c->cfg.n_kv_heads; ++h) c->len[h] += n_tokens;
  return HC_OK;
}

int headcast_packed_export(headcast_packed* c, int32_t first, int32_t n_tokens, void* k_out, void* v_out, void* stream) {
  const int rc = enter(c);
  if (rc != HC_OK) return rc;
  if (first < 0 || n_tokens < 0 || first > c->cfg.capacity - n_tokens) return fail(c, HC_ERR_INVALID_ARG, "tokens out of range");
  if ((k_out && !aligned(k_out)) || (v_out && !aligned(v_out))) return fail(c, HC_ERR_INVALID_ARG, "outputs must be 16-byte aligned device pointers");
  if (n_tokens == 0 || (!k_out && !v_out)) return HC_OK;
  const int64_t bytes = 2ll * c->cfg.n_kv_heads * n_tokens * c->cfg.head_dim;
  if ((k_out && in_storage(c, k_out, bytes)) || (v_out && in_storage(c, v_out, bytes)) || (k_out && v_out && overlap(k_out, bytes, v_out, bytes)))
    return fail(c, HC_ERR_INVALID_ARG, "an output overlaps the cache's storage or the other output");
  UnpackParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = c->view;
  p.k = static_cast<__nv_bfloat16*>(k_out);
  p.v = static_cast<__nv_bfloat16*>(v_out);
  p.n = n_tokens;
  p.first = first;
  p.len = lengths(c);
  const int rows = pack_block_tokens(c->cfg.head_dim);
  PK_CUDA(c, launch_pdl(c->cfg.head_dim == 128 ? unpack_rows_kernel<128> : unpack_rows_kernel<64>, dim3((n_tokens + rows - 1) / rows, c->cfg.n_kv_heads, 2),
                        dim3(PACK_THREADS), 0, static_cast<cudaStream_t>(stream), p));
  return HC_OK;
}

int64_t headcast_packed_workspace_bytes(const headcast_packed* c, int32_t n_queries) {
  if (!c || n_queries < 0) return HC_ERR_INVALID_ARG;
  const int64_t observe = 2ll * c->n_sm * 256 * 4;  // sums of cut pairs of token tiles
  return std::max(observe, few_rows(c, n_queries) ? RowsWorkspace(c).bytes : ManyWorkspace(c).bytes);
}

int headcast_packed_attend(headcast_packed* c, const void* q, void* out, float* lse, int32_t n_queries, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = enter(c);
  if (rc != HC_OK) return rc;
  if (n_queries < 0 || static_cast<int64_t>(n_queries) * c->cfg.n_heads > INT32_MAX - 512) return fail(c, HC_ERR_INVALID_ARG, "n_queries out of range");
  if (n_queries == 0) return HC_OK;
  if (!aligned(q) || !aligned(out)) return fail(c, HC_ERR_INVALID_ARG, "q and out must be 16-byte aligned device pointers");
  const int64_t q_bytes = 2ll * n_queries * c->cfg.n_heads * c->cfg.head_dim;
  if (q != out && overlap(q, q_bytes, out, q_bytes)) return fail(c, HC_ERR_INVALID_ARG, "out overlaps q without being q");
  if (lse && !aligned(lse, 4)) return fail(c, HC_ERR_INVALID_ARG, "lse must be 4-byte aligned");
  const int64_t lse_bytes = 4ll * n_queries * c->cfg.n_heads;
  if (lse && (overlap(lse, lse_bytes, q, q_bytes) || overlap(lse, lse_bytes, out, q_bytes))) return fail(c, HC_ERR_INVALID_ARG, "lse overlaps q or out");
  const int64_t needed = headcast_packed_workspace_bytes(c, n_queries);
  if (!aligned(workspace, 256) || workspace_bytes < needed)
    return fail(c, HC_ERR_INVALID_ARG, "the workspace must be 256-byte aligned and hold headcast_packed_workspace_bytes(%d)", n_queries);
  if (in_storage(c, out, q_bytes) || (lse && in_storage(c, lse, lse_bytes)) || in_storage(c, workspace, needed))
    return fail(c, HC_ERR_INVALID_ARG, "out, lse or the workspace overlaps the cache's storage");
  if (overlap(workspace, needed, q, q_bytes) || overlap(workspace, needed, out, q_bytes) || (lse && overlap(workspace, needed, lse, lse_bytes)))
    return fail(c, HC_ERR_INVALID_ARG, "the workspace overlaps q, out or lse");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (few_rows(c, n_queries))
    return c->cfg.head_dim == 128 ? attend_few<128>(c, q, out, lse, n_queries, workspace, st) : attend_few<64>(c, q, out, lse, n_queries, workspace, st);
  return c->cfg.head_dim == 128 ? attend_many<128>(c, q, out, lse, n_queries, workspace, st) : attend_many<64>(c, q, out, lse, n_queries, workspace, st);
}

int headcast_packed_observe(headcast_packed* c, const void* q, const float* lse, int32_t n_queries, float decay, void* workspace, int64_t workspace_bytes,
                            void* stream) {
  int rc = enter(c);
  if (rc != HC_OK) return rc;
  if (n_queries < 0 || static_cast<int64_t>(n_queries) * c->cfg.n_heads > INT32_MAX - 512) return fail(c, HC_ERR_INVALID_ARG, "n_queries out of range");
  if (!(decay >= 0.f && std::isfinite(decay))) return fail(c, HC_ERR_INVALID_ARG, "decay must be finite and not negative");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  PackedObserveParams p;
  std::memset(&p, 0, sizeof(p));
  p.c = c->view;
  p.decay = decay;
  p.len = lengths(c);
  int longest = 0;
  for (int h = 0; h < c->cfg.n_kv_heads; ++h) longest = std::max(longest, c->len[h]);
  if (longest == 0) return HC_OK;
  if (n_queries == 0) {
    if (decay != 1.f) PK_CUDA(c, launch_pdl(packed_decay_kernel, dim3((longest + 255) / 256, c->cfg.n_kv_heads), dim3(256), 0, st, p));
    return HC_OK;
  }
  if (!aligned(q)) return fail(c, HC_ERR_INVALID_ARG, "q must be a 16-byte aligned device pointer");
  if (!aligned(lse, 4)) return fail(c, HC_ERR_INVALID_ARG, "lse must be a 4-byte aligned device pointer");
  const int64_t needed = headcast_packed_workspace_bytes(c, n_queries);
  if (!aligned(workspace, 256) || workspace_bytes < needed)
    return fail(c, HC_ERR_INVALID_ARG, "the workspace must be 256-byte aligned and hold headcast_packed_workspace_bytes(%d)", n_queries);
  const int64_t q_bytes = 2ll * n_queries * c->cfg.n_heads * c->cfg.head_dim, lse_bytes = 4ll * n_queries * c->cfg.n_heads;
  if (in_storage(c, q, q_bytes) || in_storage(c, lse, lse_bytes) || in_storage(c, workspace, needed))
    return fail(c, HC_ERR_INVALID_ARG, "q, lse or the workspace overlaps the cache's storage");
  if (overlap(workspace, needed, q, q_bytes) || overlap(workspace, needed, lse, lse_bytes)) return fail(c, HC_ERR_INVALID_ARG, "the workspace overlaps q or lse");
  if (few_rows(c, n_queries)) {
    PackedObserveRowsParams r;
    std::memset(&r, 0, sizeof(r));
    r.c = c->view;
    r.q = static_cast<const __nv_bfloat16*>(q);
    r.lse = lse;
    r.n_queries = n_queries;
    r.group = c->cfg.n_heads / c->cfg.n_kv_heads;
    r.n_rows = n_queries * r.group;
    r.scale_log2e = c->scale * 1.4426950408889634f;
    r.decay = decay;
    r.len = p.len;
    // four blocks per SM, as many for every head
    const int tiles = (longest + PACK_TILE - 1) / PACK_TILE, blocks = std::min(tiles, std::max(1, 4 * c->n_sm / c->cfg.n_kv_heads));
    const bool one = r.n_rows <= 8;
    auto* rows_kernel = c->cfg.head_dim == 128 ? (one ? packed_observe_rows_kernel<128, 1> : packed_observe_rows_kernel<128, 2>)
                                               : (one ? packed_observe_rows_kernel<64, 1> : packed_observe_rows_kernel<64, 2>);
    PK_CUDA(c, launch_pdl(rows_kernel, dim3(blocks, c->cfg.n_kv_heads), dim3(OBSERVE_ROWS_THREADS), 0, st, r));
    return HC_OK;
  }
  p.lse = lse;
  p.part = static_cast<float*>(workspace);
  p.n_queries = n_queries;
  p.group = c->cfg.n_heads / c->cfg.n_kv_heads;
  p.q_tiles = (n_queries + 127) / 128;
  p.scale_log2e = c->scale * 1.4426950408889634f;
  int64_t total = 0;
  for (int h = 0; h <= PACK_MAX_HEADS; ++h) {
    p.line_first[h] = total;
    if (h < c->cfg.n_kv_heads) total += static_cast<int64_t>((c->len[h] + 255) / 256) * p.group * p.q_tiles;
  }
  p.n_cta = static_cast<int32_t>(std::min<int64_t>(c->n_sm, total));
  const uint64_t row = static_cast<uint64_t>(c->cfg.n_heads) * c->cfg.head_dim;
  if (!make_tmap_bf16_2d(&p.q_map, q, row, n_queries, row, 128)) return fail(c, HC_ERR_CUDA, "cuTensorMapEncodeTiled failed or is unavailable");
  const int smem = c->cfg.head_dim == 128 ? ObserveSmem<128>::DYN_BYTES : ObserveSmem<64>::DYN_BYTES;
  auto* kernel = c->cfg.head_dim == 128 ? packed_observe_kernel<128> : packed_observe_kernel<64>;
  rc = allow_smem(c, KERNEL_OBSERVE, kernel, smem);
  if (rc != HC_OK) return rc;
  PK_CUDA(c, launch_pdl(kernel, dim3(p.n_cta), dim3(POBS_THREADS), smem, st, p));
  if (p.n_cta > 1) PK_CUDA(c, launch_pdl(packed_observe_merge_kernel, dim3(p.n_cta - 1), dim3(256), 0, st, p));
  return HC_OK;
}

int64_t headcast_packed_evict_workspace_bytes(const headcast_packed* c) {
  if (!c) return HC_ERR_INVALID_ARG;
  return c->view.cap * c->cfg.n_kv_heads * static_cast<int64_t>(sizeof(int32_t));
}

int headcast_packed_evict(headcast_packed* c, headcast_packed* to, const int32_t* keep_host, int32_t n_first, int32_t n_recent, int32_t* index,
                          int32_t index_stride, void* workspace, int64_t workspace_bytes, void* stream) {
  const int rc = enter(c);
  if (rc != HC_OK) return rc;
  const int n_kv = c->cfg.n_kv_heads, d = c->cfg.head_dim;
  if (!to || to == c || !keep_host) return fail(c, HC_ERR_INVALID_ARG, "another cache and a number of tokens per head are needed");
  if (to->cfg.n_kv_heads != n_kv || to->cfg.head_dim != d || to->device != c->device)
    return fail(c, HC_ERR_INVALID_ARG, "the other cache has other key/value heads, another head_dim or another device");
  if (in_storage(c, to->view.status, to->bytes)) return fail(c, HC_ERR_INVALID_ARG, "the caches share storage");
  if (n_first < 0 || n_recent < 0) return fail(c, HC_ERR_INVALID_ARG, "n_first and n_recent must not be negative");
  SelectParams s;
  std::memset(&s, 0, sizeof(s));
  s.len = lengths(c);
  int longest = 0, most = 0;
  for (int h = 0; h < n_kv; ++h) {
    if (keep_host[h] < 0) return fail(c, HC_ERR_INVALID_ARG, "a head's number of tokens must not be negative");
    s.keep.n[h] = std::min(keep_host[h], c->len[h]);
    if (s.keep.n[h] > to->cfg.capacity) return fail(c, HC_ERR_STATE, "head %d would move %d tokens, the other cache holds at most %d", h, s.keep.n[h], to->cfg.capacity);
    longest = std::max(longest, c->len[h]);
    most = std::max(most, s.keep.n[h]);
  }
  if (index && (!aligned(index, 4) || index_stride < most)) return fail(c, HC_ERR_INVALID_ARG, "index must be 4-byte aligned with rows of at least %d", most);
  if (most > 0 && !index && (!aligned(workspace, 256) || workspace_bytes < headcast_packed_evict_workspace_bytes(c)))
    return fail(c, HC_ERR_INVALID_ARG, "the workspace must be 256-byte aligned and hold headcast_packed_evict_workspace_bytes()");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (most > 0) {
    const void* places = index ? index : workspace;
    const int64_t bytes = index ? 4 * (static_cast<int64_t>(index_stride) * (n_kv - 1) + most) : headcast_packed_evict_workspace_bytes(c);
    if (in_storage(c, places, bytes) || in_storage(to, places, bytes)) return fail(c, HC_ERR_INVALID_ARG, "the index or the workspace overlaps a cache's storage");
    s.weights = c->view.weights;
    s.index = index ? index : static_cast<int32_t*>(workspace);
    s.index_stride = index ? index_stride : c->view.cap;
    s.cap = c->view.cap;
    s.n_first = n_first;
    s.n_recent = n_recent;
    // Blocks per head, 4096 tokens each: selection and move of 9000 tokens, 12 heads of 128, 14.7 us with four and 17.2 with one, 12000
    // 15.7 / 20.3, 5000 11.7-13.1 with two or one; with eight blocks 1000 tokens took 1.6 us more than with a cluster of one.
    int blocks = 1;
    while (blocks < SELECT_MAX_BLOCKS && blocks * 4096 < longest) blocks *= 2;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(blocks * n_kv);
    lc.blockDim = dim3(SELECT_THREADS);
    lc.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = blocks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    lc.attrs = attr;
    lc.numAttrs = 2;
    PK_CUDA(c, cudaLaunchKernelEx(&lc, blocks == 1 ? evict_select_kernel<true> : evict_select_kernel<false>, s));
    EvictMoveParams m;
    std::memset(&m, 0, sizeof(m));
    m.src = c->view;
    m.dst = to->view;
    m.index = s.index;
    m.index_stride = s.index_stride;
    m.keep = s.keep;
    const int tokens = EVICT_MOVE_THREADS / (d / 16);
    PK_CUDA(c, launch_pdl(d == 128 ? evict_move_kernel<128> : evict_move_kernel<64>, dim3((most + tokens - 1) / tokens, n_kv), dim3(EVICT_MOVE_THREADS), 0, st, m));
  }
  for (int h = 0; h < n_kv; ++h) to->len[h] = s.keep.n[h];
  return HC_OK;
}

int headcast_packed_check(headcast_packed* c, void* stream) {
  const int rc = enter(c);
  if (rc != HC_OK) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t status = 0;
  PK_CUDA(c, cudaMemcpyAsync(&status, c->view.status, sizeof(status), cudaMemcpyDeviceToHost, st));
  PK_CUDA(c, cudaStreamSynchronize(st));
  if (status == 0) return HC_OK;
  PK_CUDA(c, cudaMemsetAsync(c->view.status, 0, sizeof(int32_t), st));
  return fail(c, HC_ERR_TIMEOUT, "a kernel gave up on a bounded wait (site %d)", status);
}

}  // extern "C"
