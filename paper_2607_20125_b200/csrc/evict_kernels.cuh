// Eviction from a packed cache: which tokens of a head stay, and their move into another cache.
//
// evict_select_kernel, one cluster of up to 8 blocks per head: the keep-th largest weight by radix selection (up to three digits
// of 11, 11 and 10 bits of an order-preserving integer), then the places of all tokens above it, and of the first ones equal to it, in
// order.  The blocks of a cluster split the head's tokens, a warp a run of them; each block finds the digit for itself from the
// histograms of all, first among 64 sums of 32 bins, then among that group's bins, so that little crosses between the blocks (all
// 2048 bins read from all blocks took 2.7 us a digit).  Counts are integers and places follow from prefix sums, so the result is
// the same every time.  What it costs is latency: the weights are read once, into registers (again from L2 where a thread's share
// exceeds SELECT_HELD), and a handful of cluster barriers follow one another.
// evict_move_kernel copies the rows: bound by memory, 148 bytes read and written per token at d = 128.
#pragma once
#include "packed_format.cuh"

namespace hc {

constexpr int SELECT_THREADS = 1024;
constexpr int SELECT_HELD = 12;   // keys that a thread keeps in registers
constexpr int SELECT_BINS = 2048, SELECT_GROUPS = 64;

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
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// A word of another block's shared memory, at the place where `p` is in this one's.
__device__ __forceinline__ uint32_t peer_word(const uint32_t* p, uint32_t rank) {
  uint32_t at, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
constexpr int SELECT_MAX_BLOCKS = 8;  // of a cluster

// Of n counts (64 or 32, two or one per lane of the first warp), highest first: which one holds the k-th key, the rank in it, and the
// count.  The whole block calls it; the counts lie in `sums`, the answer goes to `found`.  Its barriers also keep the counts of one call
// from the reads of the one before, and the answers likewise.
template <int N>
__device__ __forceinline__ void find_kth(const uint32_t* sums, uint32_t k, uint32_t* found) {
  const int tid = threadIdx.x;
  __syncthreads();
  if (tid < 32) {
    constexpr int PER = N / 32;
    uint32_t c[PER], total = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) total += c[i] = sums[tid * PER + i];
    uint32_t suffix = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_down_sync(0xffffffffu, suffix, o);
      if (tid + o < 32) suffix += up;
    }
    uint32_t above = suffix - total;
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      if (above < k && k <= above + c[i]) {  // exactly one lane, once
        found[0] = tid * PER + i;
        found[1] = k - above;
        found[2] = c[i];
      }
      above += c[i];
    }
  }
  __syncthreads();
}

// ONE: clusters of one block, whose barriers and reads are the block's own (3003 tokens of 6 heads, selection and move: 9.7 us, as a cluster 11.7).
template <bool ONE>
__global__ void __launch_bounds__(SELECT_THREADS) evict_select_kernel(const __grid_constant__ SelectParams p) {
  __shared__ uint32_t hist[2][SELECT_BINS], groups[2][SELECT_GROUPS];  // used in turn: one cluster barrier per digit
  __shared__ uint32_t sums[SELECT_GROUPS], found[3], counts[2], warp_gt[32], warp_eq[32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t rank = ONE ? 0u : cluster_rank(), ranks = ONE ? 1u : cluster_size();
  auto sync_all = [] { ONE ? __syncthreads() : cluster_sync(); };
  auto word_of = [](const uint32_t* p, uint32_t rank) { return ONE ? *p : peer_word(p, rank); };
  const int h = blockIdx.x / ranks;
  const int n = p.len.n[h], keep = p.keep.n[h];
  pdl_launch_dependents();
  for (int b = tid; b < 2 * SELECT_BINS; b += SELECT_THREADS) (&hist[0][0])[b] = 0;
  pdl_wait();
  if (keep <= 0) return;  // the same for the whole cluster
  const int lo = static_cast<int>(static_cast<long long>(n) * rank / ranks), hi = static_cast<int>(static_cast<long long>(n) * (rank + 1) / ranks);
  const float* w = p.weights + static_cast<size_t>(h) * p.cap;
  const int recent = max(p.n_first, n - p.n_recent);  // tokens from here on always stay, and those before n_first
  // a warp's run of tokens, 32 at a time
  const int rounds = (hi - lo + SELECT_THREADS - 1) / SELECT_THREADS;
  const int first = lo + warp * rounds * 32 + lane;
  auto from_memory = [&](int j) {
    const int i = first + 32 * j;
    return i < hi ? select_key(w[i], i < p.n_first || i >= recent) : 0u;
  };
  uint32_t held[SELECT_HELD];
  if (rounds <= SELECT_HELD) {
    float raw[SELECT_HELD];
#pragma unroll
    for (int j = 0; j < SELECT_HELD; ++j) raw[j] = j < rounds && first + 32 * j < hi ? w[first + 32 * j] : 0.f;
#pragma unroll
    for (int j = 0; j < SELECT_HELD; ++j) {
      const int i = first + 32 * j;
      held[j] = i < hi ? select_key(raw[j], i < p.n_first || i >= recent) : 0u;
    }
  }
  // f(j, key of token first + 32 j, whether there is one), round by round, the whole warp together
  auto each = [&](auto&& f) {
    if (rounds <= SELECT_HELD) {
#pragma unroll
      for (int j = 0; j < SELECT_HELD; ++j)
        if (j < rounds) f(j, held[j], first + 32 * j < hi);
    } else {
#pragma unroll 1
      for (int j = 0; j < rounds; ++j) f(j, from_memory(j), first + 32 * j < hi);
    }
  };

  __syncthreads();
  uint32_t prefix = 0, mask = 0, k = keep;  // the k-th largest of the keys that agree with prefix under mask
#pragma unroll 1
  for (int digit = 0; digit < 3; ++digit) {
    const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
    uint32_t* mine = hist[digit & 1];
    each([&](int, uint32_t key, bool there) {
      const bool counts_in = there && (key & mask) == prefix;
      // Equal weights are common (tokens that nothing has looked at yet), and a warp of them would add to one bin 32 times in turn:
      // the lanes that agree with the first that counts add once.
      const uint32_t in = __ballot_sync(0xffffffffu, counts_in);
      if (in == 0) return;
      const uint32_t bin = (key >> shift) & ((1u << bits) - 1u);
      const int chosen = __ffs(in) - 1;
      const uint32_t chosen_bin = __shfl_sync(0xffffffffu, bin, chosen);  // (by every lane, also those that do not count)
      const bool like = counts_in && bin == chosen_bin;
      const uint32_t same = __ballot_sync(0xffffffffu, like);
      if (lane == chosen) atomicAdd(&mine[bin], static_cast<uint32_t>(__popc(same)));
      else if (counts_in && !like) atomicAdd(&mine[bin], 1u);
    });
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // a warp sums two groups of 32 bins
      const uint32_t sum = __reduce_add_sync(0xffffffffu, mine[(2 * warp + x) * 32 + lane]);
      if (lane == 0) groups[digit & 1][2 * warp + x] = sum;
    }
    sync_all();
    if (digit == 1)  // the first digit's bins are the third's; all blocks have read them
      for (int b = tid; b < SELECT_BINS; b += SELECT_THREADS) hist[0][b] = 0;
    // eight lanes per group, and then per bin: one for each block
    if (tid < 8 * SELECT_GROUPS) {
      uint32_t c = (tid & 7) < ranks ? word_of(&groups[digit & 1][tid >> 3], tid & 7) : 0u;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if ((tid & 7) == 0) sums[tid >> 3] = c;
    }
    find_kth<SELECT_GROUPS>(sums, k, found);
    const uint32_t group = found[0];
    k = found[1];
    if (tid < 8 * 32) {
      uint32_t c = (tid & 7) < ranks ? word_of(&mine[group * 32 + (tid >> 3)], tid & 7) : 0u;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
      if ((tid & 7) == 0) sums[tid >> 3] = c;
    }
    find_kth<32>(sums, k, found);
    prefix |= (group * 32 + found[0]) << shift;
    mask |= ((1u << bits) - 1u) << shift;
    k = found[1];
    if (k == found[2]) break;  // all of that bin stay (in most cases it holds one key by the second digit)
  }
  // `prefix` is the keep-th largest key, and k tokens of that key stay: the first ones.  (Or all keys from `prefix` on stay.)
  uint32_t n_gt = 0, n_eq = 0;
  each([&](int, uint32_t key, bool there) {
    n_gt += __popc(__ballot_sync(0xffffffffu, there && key > prefix));
    n_eq += __popc(__ballot_sync(0xffffffffu, there && key == prefix));
  });
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
  sync_all();
  // of the tokens before this warp's: those of the blocks before, then of the warps before
  uint32_t gt = 0, eq = 0;
  if (lane < rank) {
    gt = word_of(&counts[0], lane);
    eq = word_of(&counts[1], lane);
  }
  if (lane < warp) {
    gt += warp_gt[lane];
    eq += warp_eq[lane];
  }
  gt = __reduce_add_sync(0xffffffffu, gt);
  eq = __reduce_add_sync(0xffffffffu, eq);
  int32_t* out = p.index + static_cast<size_t>(h) * p.index_stride;
  const uint32_t before = (1u << lane) - 1u;
  each([&](int j, uint32_t key, bool there) {
    const bool is_gt = there && key > prefix, is_eq = there && key == prefix;
    const uint32_t m_gt = __ballot_sync(0xffffffffu, is_gt), m_eq = __ballot_sync(0xffffffffu, is_eq);
    const uint32_t my_gt = gt + __popc(m_gt & before), my_eq = eq + __popc(m_eq & before);
    if (is_gt || (is_eq && my_eq < k)) out[my_gt + min(my_eq, k)] = first + 32 * j;
    gt += __popc(m_gt);
    eq += __popc(m_eq);
  });
  if (!ONE) cluster_sync();  // no block leaves while another may read its shared memory
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
