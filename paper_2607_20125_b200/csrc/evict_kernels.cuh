// Eviction from a packed cache: which tokens of a head stay, and their move into another cache.
//
// evict_select_kernel, one cluster of up to 8 blocks per head: the keep-th largest weight by radix selection (three digits of
// 11, 11 and 10 bits of an order-preserving integer), then the places of all tokens above it, and of the first ones equal to it, in
// order.  The blocks of a cluster split the head's tokens, add up their histograms through each other's shared memory, and each finds
// the digit for itself.  Counts are integers and places follow from prefix sums, so the result is the same every time.
// What it costs is latency: 4 bytes per token are read once from memory (again from L2 where a block's share exceeds
// SELECT_KEYS), and a handful of cluster barriers follow one another.
// evict_move_kernel copies the rows: bound by memory, 148 bytes read and written per token at d = 128.
#pragma once
#include "packed_format.cuh"

namespace hc {

constexpr int SELECT_THREADS = 1024;
constexpr int SELECT_KEYS = 24576;  // keys that a block keeps in shared memory
constexpr int SELECT_BINS = 2048;
constexpr int SELECT_SMEM = SELECT_KEYS * 4 + 2 * SELECT_BINS * 4;

struct SelectParams {
  const float* weights;  // [n_kv][cap]
  int32_t* index;        // [n_kv][index_stride]
  int64_t cap, index_stride;
  int32_t n_first, n_recent;
  HeadCounts len, keep;  // keep <= len
};

// Larger weights have larger keys; -0 equals 0, a NaN is below everything, a token that always stays above.
__device__ __forceinline__ uint32_t select_key(float w, bool always) {
  if (always) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w == 0.f ? 0.f : w);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Two words of another block's shared memory, at the place where `p` is in this one's.
__device__ __forceinline__ uint2 peer_words(const uint32_t* p, uint32_t rank) {
  uint32_t at;
  uint2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at) : "memory");
  return v;
}
constexpr int SELECT_MAX_BLOCKS = 8;  // of a cluster

__global__ void __launch_bounds__(SELECT_THREADS) evict_select_kernel(const __grid_constant__ SelectParams p) {
  extern __shared__ uint32_t select_smem[];
  uint32_t* const keys = select_smem;
  uint32_t* const hist = select_smem + SELECT_KEYS;  // two histograms, used in turn: one cluster barrier per digit
  __shared__ uint32_t warp_sum[32], found[2], warp_gt[32], warp_eq[32];
  __shared__ alignas(8) uint32_t counts[2];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = cluster_rank(), ranks = cluster_size();
  const int h = blockIdx.x / ranks;
  const int n = p.len.n[h], keep = p.keep.n[h];
  pdl_launch_dependents();
  pdl_wait();
  if (keep <= 0) return;  // the same for the whole cluster
  const int lo = static_cast<int>(static_cast<long long>(n) * rank / ranks), hi = static_cast<int>(static_cast<long long>(n) * (rank + 1) / ranks);
  const float* w = p.weights + static_cast<size_t>(h) * p.cap;
  const int recent = max(p.n_first, n - p.n_recent);  // tokens from here on always stay, and those before n_first
  const bool held = hi - lo <= SELECT_KEYS;
  auto from_memory = [&](int i) { return select_key(w[i], i < p.n_first || i >= recent); };
  auto key_at = [&](int i) { return held ? keys[i - lo] : from_memory(i); };
  if (held)
    for (int i = lo + tid; i < hi; i += SELECT_THREADS) keys[i - lo] = from_memory(i);

  uint32_t prefix = 0, mask = 0, k = keep;  // the k-th largest of the keys that agree with prefix under mask
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    uint32_t* mine = hist + (digit & 1) * SELECT_BINS;
    for (int b = tid; b < SELECT_BINS; b += SELECT_THREADS) mine[b] = 0;
    __syncthreads();
    for (int i0 = lo + warp * 32; i0 < hi; i0 += SELECT_THREADS) {
      const int i = i0 + lane;
      const uint32_t key = i < hi ? key_at(i) : 0u;
      const bool counts_in = i < hi && (key & mask) == prefix;
      const uint32_t bin = counts_in ? (key >> shift) & ((1u << bits) - 1u) : 0xffffffffu;
      // lanes of one bin add once: weights crowd into few bins, and equal ones (tokens that nothing has looked at yet) into one
      const uint32_t same = __match_any_sync(0xffffffffu, bin);
      if (counts_in && lane == __ffs(same) - 1) atomicAdd(&mine[bin], static_cast<uint32_t>(__popc(same)));
    }
    cluster_sync();
    // each thread owns two bins; how many keys lie in higher bins is a suffix sum over threads
    uint32_t c0 = 0, c1 = 0;
    uint2 theirs[SELECT_MAX_BLOCKS];
#pragma unroll
    for (uint32_t x = 0; x < SELECT_MAX_BLOCKS; ++x) theirs[x] = x < ranks ? peer_words(&mine[2 * tid], x) : make_uint2(0, 0);
#pragma unroll
    for (uint32_t x = 0; x < SELECT_MAX_BLOCKS; ++x) {
      c0 += theirs[x].x;
      c1 += theirs[x].y;
    }
    uint32_t suffix = c0 + c1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_down_sync(0xffffffffu, suffix, o);
      if (lane + o < 32) suffix += up;
    }
    if (lane == 0) warp_sum[warp] = suffix;
    __syncthreads();
    const uint32_t above = suffix - (c0 + c1) + __reduce_add_sync(0xffffffffu, lane > warp ? warp_sum[lane] : 0u);
    if (above < k && k <= above + c0 + c1) {  // exactly one thread
      const bool upper = k <= above + c1;
      found[0] = 2 * tid + (upper ? 1 : 0);
      found[1] = k - (upper ? above : above + c1);
    }
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= ((1u << bits) - 1u) << shift;
    k = found[1];
  }
  // `prefix` is the keep-th largest key, and k tokens of that key stay: the first ones.  Each warp takes a run of tokens.
  const int per_warp = (hi - lo + 31) / 32;
  const int a = min(hi, lo + warp * per_warp), b = min(hi, a + per_warp);
  uint32_t n_gt = 0, n_eq = 0;
  for (int i0 = a; i0 < b; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t key = i < b ? key_at(i) : 0u;
    n_gt += __popc(__ballot_sync(0xffffffffu, i < b && key > prefix));
    n_eq += __popc(__ballot_sync(0xffffffffu, i < b && key == prefix));
  }
  if (lane == 0) {
    warp_gt[warp] = n_gt;
    warp_eq[warp] = n_eq;
  }
  __syncthreads();
  if (warp == 0) {
    const uint32_t g = __reduce_add_sync(0xffffffffu, warp_gt[lane]), e = __reduce_add_sync(0xffffffffu, warp_eq[lane]);
    if (lane == 0) {
      counts[0] = g;
      counts[1] = e;
    }
  }
  cluster_sync();
  // of the tokens before this warp's: those of the blocks before, then of the warps before
  uint2 before_me = make_uint2(0, 0);
  if (lane < rank) before_me = peer_words(counts, lane);
  if (lane < warp) {
    before_me.x += warp_gt[lane];
    before_me.y += warp_eq[lane];
  }
  uint32_t gt = __reduce_add_sync(0xffffffffu, before_me.x), eq = __reduce_add_sync(0xffffffffu, before_me.y);
  int32_t* out = p.index + static_cast<size_t>(h) * p.index_stride;
  for (int i0 = a; i0 < b; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t key = i < b ? key_at(i) : 0u;
    const bool is_gt = i < b && key > prefix, is_eq = i < b && key == prefix;
    const uint32_t m_gt = __ballot_sync(0xffffffffu, is_gt), m_eq = __ballot_sync(0xffffffffu, is_eq);
    const uint32_t before = (1u << lane) - 1u;
    const uint32_t my_gt = gt + __popc(m_gt & before), my_eq = eq + __popc(m_eq & before);
    if (is_gt || (is_eq && my_eq < k)) out[my_gt + min(my_eq, k)] = i;
    gt += __popc(m_gt);
    eq += __popc(m_eq);
  }
  cluster_sync();  // no block leaves while another may read its shared memory
}

struct EvictMoveParams {
  PackedView src, dst;
  const int32_t* index;
  int64_t index_stride;
  HeadCounts keep;
};
constexpr int EVICT_MOVE_THREADS = 256;

// D / 16 threads copy a token: each 16 bytes of codes, and every quarter of them the scales or the weight.
template <int D>
__global__ void __launch_bounds__(EVICT_MOVE_THREADS) evict_move_kernel(const __grid_constant__ EvictMoveParams p) {
  constexpr int LANES = D / 16, HALF = LANES / 2;
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.y, u = threadIdx.x % LANES;
  const int j = blockIdx.x * (EVICT_MOVE_THREADS / LANES) + threadIdx.x / LANES;
  if (j >= p.keep.n[h]) return;
  const size_t from = static_cast<size_t>(h) * p.src.cap + p.index[static_cast<size_t>(h) * p.index_stride + j];
  const size_t to = static_cast<size_t>(h) * p.dst.cap + j;
  const bool is_v = u >= HALF;
  const int part = u % HALF;
  const uint4 codes = *(reinterpret_cast<const uint4*>((is_v ? p.src.v_codes : p.src.k_codes) + from * (D / 2)) + part);
  using Scales = typename std::conditional<D == 128, uint2, uint32_t>::type;
  Scales scales{};
  float weight = 0.f;
  if (part == 0) scales = *reinterpret_cast<const Scales*>((is_v ? p.src.v_scales : p.src.k_scales) + from * (D / PACK_GROUP));
  if (u == 1) weight = p.src.weights[from];
  *(reinterpret_cast<uint4*>((is_v ? p.dst.v_codes : p.dst.k_codes) + to * (D / 2)) + part) = codes;
  if (part == 0) *reinterpret_cast<Scales*>((is_v ? p.dst.v_scales : p.dst.k_scales) + to * (D / PACK_GROUP)) = scales;
  if (u == 1) p.dst.weights[to] = weight;
}

}  // namespace hc
