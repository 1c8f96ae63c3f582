// How much attention every token of a packed cache receives: weight_j = decay * weight_j + sum over query rows i of
// exp(scale * q_i . k_j - lse_i), with the log-sum-exps that the attention returned.
//
// Only logits are needed, and sums over queries: so the product is turned around, S^T = K Q^T, tokens on the 128 lanes of tensor
// memory and queries in its columns.  Two threads own a token and add up half its columns each in registers.  A work item is a pair of
// token tiles (256 tokens) of one key/value head, converted to bf16 (exact) once and kept in shared memory, over a range of
// query tiles that arrive by TMA as the caller left them.  Items are laid end to end and cut into equal shares like
// those of packed_attn_kernel; sums of cut items are joined in the order of the line, so results do not vary from run to run.
//   warp 0 issues products, warp 1 loads query tiles, warps 2 and 3 their log-sum-exps, warps 4-7 convert the next pair of
//   tiles while this one is in use, warps 8-23 add up: four per scheduler, since with two (a thread per token) the loop waited for its own
//   latencies, 3300 clk a step.
// What bounds it: latency.  One exponential per logit, 2 * 128 * 128 per step, would be 2048 clk of the special-function unit beside 1024 clk of
// products; a quarter of the exponentials is evaluated on the FMA pipe (none to a half of them: level to 20 % slower).  A step takes 2700 clk,
// the unit busy 57 % of them: a warp waits for each of its loads from tensor memory right behind its issue.  4680 queries x 32760 tokens,
// 12 heads of 128: 543 us, and 620 for seconds on end, at the power cap.
#pragma once
#include "packed_attn_kernel.cuh"

namespace hc {

constexpr int POBS_THREADS = 768;
constexpr int POBS_LSE_SLOTS = 4;
constexpr int POBS_POLY_MASK = 1;  // every other group of four columns has two of them take the polynomial
constexpr float WEIGHS_NOTHING = -1e30f;

struct PackedObserveParams {
  PackedView c;
  const float* lse;   // [n_kv * group][n_queries]
  float* part;        // [2 * n_cta][256], slots as in PackedAttnParams
  int32_t n_queries, group, q_tiles;  // q_tiles = ceil(n_queries / 128)
  int32_t n_cta;
  float scale_log2e, decay;
  int64_t line_first[PACK_MAX_HEADS + 1];  // steps of the heads before h: pairs of token tiles times group * q_tiles
  HeadCounts len;
  alignas(64) CUtensorMap q_map;  // [n_queries][n_heads * d] bf16, boxes of 64 columns and 128 rows
};

struct ObserveItem {
  int32_t head, pair, begin, end, slot;  // query tiles [begin, end) of group * q_tiles
};
__host__ __device__ inline ObserveItem observe_item(const PackedObserveParams& p, int cta, int64_t& x, int64_t hi, int& head) {
  while (p.line_first[head + 1] <= x) ++head;
  const int steps = p.group * p.q_tiles;
  ObserveItem w;
  w.head = head;
  const int64_t in_head = x - p.line_first[head];
  w.pair = static_cast<int32_t>(in_head / steps);
  w.begin = static_cast<int32_t>(in_head - static_cast<int64_t>(w.pair) * steps);
  const int64_t end = w.begin + (hi - x);
  w.end = end < steps ? static_cast<int32_t>(end) : steps;
  x += w.end - w.begin;
  w.slot = w.begin > 0 ? 2 * cta : w.end < steps ? 2 * cta + 1 : -1;
  return w;
}

template <int D>
struct ObserveSmem {
  static constexpr int BLOCK_BYTES = 128 * 128;
  static constexpr int TILE_BYTES = (D / 64) * BLOCK_BYTES;
  static constexpr int Q_SLOTS = D == 128 ? 2 : 4;
  static constexpr int Q_OFF = 4 * TILE_BYTES;  // two pairs of token tiles, then the ring of query tiles
  static constexpr int LSE_OFF = Q_OFF + Q_SLOTS * TILE_BYTES;
  static constexpr int DYN_BYTES = LSE_OFF + POBS_LSE_SLOTS * 128 * 4 + 1024;
};

template <int D>
__global__ void __launch_bounds__(POBS_THREADS, 1) packed_observe_kernel(const __grid_constant__ PackedObserveParams p) {
  using SM = ObserveSmem<D>;
  constexpr uint32_t TMEM_COLS = 512;  // two buffers of two 128-column products
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = aligned_shared<1024>(smem_raw);
  __shared__ uint64_t bar_k_full[2], bar_k_free[2], bar_q_full[SM::Q_SLOTS], bar_q_free[SM::Q_SLOTS], bar_l_full[POBS_LSE_SLOTS], bar_l_free[POBS_LSE_SLOTS],
      bar_s_full[2], bar_s_free[2];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ float other_half[256];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bar_k_full[i], 4);
      mbar_init(&bar_k_free[i], 1);
      mbar_init(&bar_s_full[i], 1);
      mbar_init(&bar_s_free[i], 16);
    }
    for (int i = 0; i < SM::Q_SLOTS; ++i) {
      mbar_init(&bar_q_full[i], 1);
      mbar_init(&bar_q_free[i], 1);
    }
    for (int i = 0; i < POBS_LSE_SLOTS; ++i) {
      mbar_init(&bar_l_full[i], 2);
      mbar_init(&bar_l_free[i], 16);
    }
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&tmem_slot, TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  // All of the above runs while the kernel before drains.
  pdl_launch_dependents();
  pdl_wait();
  const uint32_t tmem = tmem_slot;
  volatile int* abortp = &abort_flag;
  const int64_t total = p.line_first[p.c.n_kv];
  int64_t x = share_begin(blockIdx.x, total, p.n_cta);
  const int64_t x_hi = share_begin(blockIdx.x + 1, total, p.n_cta);
  int head = 0;
  float* const lse_ring = reinterpret_cast<float*>(smem + SM::LSE_OFF);

  if (warp == 0) {
    // ------------------------------------------------------------------ products (the whole warp, converged)
    const uint32_t elected = elect_one();
    const uint32_t idesc = idesc_bf16_f32(128, 128, 0, 0);
    const uint64_t k_desc = smem_desc_sw128(smem_u32(smem), 16, 1024), q_desc = smem_desc_sw128(smem_u32(smem + SM::Q_OFF), 16, 1024);
    uint32_t item = 0, step = 0;
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity, int code) -> bool { return mbar_wait_warp(bar, parity, abortp, p.c.status, code); };
    while (ok && x < x_hi) {
      const ObserveItem w = observe_item(p, blockIdx.x, x, x_hi, head);
      const bool two = p.len.n[w.head] - w.pair * 256 > 128;
      const uint32_t kb = item & 1;
      if (!(ok = wait(&bar_k_full[kb], (item >> 1) & 1, 101))) break;
      ++item;
      for (int s = w.begin; s < w.end; ++s, ++step) {
        const uint32_t st = step % SM::Q_SLOTS, buf = step & 1;
        if (!(ok = wait(&bar_q_full[st], (step / SM::Q_SLOTS) & 1, 102))) break;
        if (!(ok = wait(&bar_s_free[buf], ((step >> 1) & 1) ^ 1, 103))) break;
        tc_fence_after_sync();
        const uint64_t q_at = q_desc + ((st * SM::TILE_BYTES) >> 4), k_at = k_desc + ((2 * kb * SM::TILE_BYTES) >> 4);
        mma_block_ss<D / 16>(tmem + buf * 256, k_at, q_at, idesc, SM::BLOCK_BYTES >> 4, elected);
        if (two) mma_block_ss<D / 16>(tmem + buf * 256 + 128, k_at + (SM::TILE_BYTES >> 4), q_at, idesc, SM::BLOCK_BYTES >> 4, elected);
        mma_commit(&bar_s_full[buf], elected);
        mma_commit(&bar_q_free[st], elected);
      }
      mma_commit(&bar_k_free[kb], elected);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ query tiles
    if (lane == 0) {
      uint32_t step = 0;
      bool ok = true;
      const uint64_t policy = l2_policy_evict_last();  // every pair of token tiles of the head reads them again
      while (ok && x < x_hi) {
        const ObserveItem w = observe_item(p, blockIdx.x, x, x_hi, head);
        for (int s = w.begin; s < w.end; ++s, ++step) {
          const uint32_t st = step % SM::Q_SLOTS;
          if (!(ok = mbar_wait(&bar_q_free[st], ((step / SM::Q_SLOTS) & 1) ^ 1, abortp, p.c.status, 104))) break;
          mbar_arrive_expect_tx(&bar_q_full[st], SM::TILE_BYTES);
          const int g = s / p.q_tiles, row = (s - g * p.q_tiles) * 128;
          for (int b = 0; b < D / 64; ++b)
            tma_load_2d_hint(smem + SM::Q_OFF + st * SM::TILE_BYTES + b * SM::BLOCK_BYTES, &p.q_map, (w.head * p.group + g) * D + 64 * b, row, &bar_q_full[st], policy);
        }
      }
      if (!ok) {
        for (uint32_t back = 1; back <= SM::Q_SLOTS && back <= step; ++back) {  // the copies in flight land before the block leaves
          int local_abort = 0;
          mbar_wait(&bar_q_full[(step - back) % SM::Q_SLOTS], ((step - back) / SM::Q_SLOTS) & 1, &local_abort, p.c.status, 105);
        }
      }
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------------ log-sum-exps, negated and in the log2 domain: two queries per lane
    uint32_t step = 0;
    bool ok = true;
    const int at = (warp - 2) * 64 + 2 * lane;
    while (ok && x < x_hi) {
      const ObserveItem w = observe_item(p, blockIdx.x, x, x_hi, head);
      for (int s = w.begin; s < w.end; ++s, ++step) {
        const uint32_t st = step % POBS_LSE_SLOTS;
        const int g = s / p.q_tiles, t = (s - g * p.q_tiles) * 128 + at;
        const float* src = p.lse + static_cast<size_t>(w.head * p.group + g) * p.n_queries + t;
        // Queries behind the last weigh nothing, nor does one with a log-sum-exp of infinity: far below every logit, but finite
        // (see the polynomial).  A NaN stays one.
        float2 v;
        v.x = t < p.n_queries ? -1.4426950408889634f * src[0] : WEIGHS_NOTHING;
        v.y = t + 1 < p.n_queries ? -1.4426950408889634f * src[1] : WEIGHS_NOTHING;
        v.x = v.x < WEIGHS_NOTHING ? WEIGHS_NOTHING : v.x > -WEIGHS_NOTHING ? -WEIGHS_NOTHING : v.x;
        v.y = v.y < WEIGHS_NOTHING ? WEIGHS_NOTHING : v.y > -WEIGHS_NOTHING ? -WEIGHS_NOTHING : v.y;
        if (!(ok = mbar_wait_warp(&bar_l_free[st], ((step / POBS_LSE_SLOTS) & 1) ^ 1, abortp, p.c.status, 106))) break;
        *reinterpret_cast<float2*>(lse_ring + st * 128 + at) = v;
        __syncwarp();
        mbar_arrive_if(&bar_l_full[st], lane == 0);
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------------ conversion: a thread takes one token of each tile
    const int row = tid - 128;
    uint32_t item = 0;
    bool ok = true;
    while (ok && x < x_hi) {
      const ObserveItem w = observe_item(p, blockIdx.x, x, x_hi, head);
      const bool two = p.len.n[w.head] - w.pair * 256 > 128;
      const uint32_t kb = item & 1;
      const size_t first = static_cast<size_t>(w.head) * p.c.cap + static_cast<size_t>(w.pair) * 256 + row;
      uint4 codes[2][D / 32];
      uint32_t scales[2][D / 64];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t && !two) continue;
        const uint4* src = reinterpret_cast<const uint4*>(p.c.k_codes + (first + t * 128) * (D / 2));
        const uint32_t* sc = reinterpret_cast<const uint32_t*>(p.c.k_scales + (first + t * 128) * (D / PACK_GROUP));
#pragma unroll
        for (int i = 0; i < D / 32; ++i) codes[t][i] = src[i];
#pragma unroll
        for (int i = 0; i < D / 64; ++i) scales[t][i] = sc[i];
      }
      if (!(ok = mbar_wait_warp(&bar_k_free[kb], ((item >> 1) & 1) ^ 1, abortp, p.c.status, 107))) break;
      ++item;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t && !two) continue;
        uint8_t* dst = smem + (2 * kb + t) * SM::TILE_BYTES;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
          const uint32_t words[4] = {codes[t][i].x, codes[t][i].y, codes[t][i].z, codes[t][i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int chunk = 4 * i + k;
            uint32_t v[4];
            word_to_bf16x2(words[k], scale_value(scales[t][chunk / 8], (chunk / 2) % 4), v);
            *reinterpret_cast<uint4*>(dst + (chunk / 8) * SM::BLOCK_BYTES + sw128_offset(row, chunk % 8)) = make_uint4(v[0], v[1], v[2], v[3]);
          }
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      mbar_arrive_if(&bar_k_full[kb], lane == 0);
    }
  } else {
    // ------------------------------------------------------------------ sums: two threads per token, half of a tile's columns each
    const int t = ((warp - 8) >> 2) & 1, r = ((warp & 3) << 5) | lane, half = (warp - 8) >> 3;
    const uint32_t s_addr = tmem + (static_cast<uint32_t>((warp & 3) << 5) << 16) + t * 128 + half * 64;
    const uint64_t c2 = pack_f32x2(p.scale_log2e, p.scale_log2e);
    uint32_t step = 0;
    bool ok = true;
    while (x < x_hi) {
      const ObserveItem w = observe_item(p, blockIdx.x, x, x_hi, head);
      const int token = w.pair * 256 + t * 128 + r;
      const bool tile_there = p.len.n[w.head] - w.pair * 256 > t * 128;
      float sum = 0.f;
      for (int s = w.begin; s < w.end; ++s, ++step) {
        const uint32_t st = step % POBS_LSE_SLOTS, buf = step & 1;
        if (ok) ok = mbar_wait_warp(&bar_l_full[st], (step / POBS_LSE_SLOTS) & 1, abortp, p.c.status, 108);
        if (ok) ok = mbar_wait_warp(&bar_s_full[buf], (step >> 1) & 1, abortp, p.c.status, 109);
        if (!ok) break;
        tc_fence_after_sync();
        const int columns = min(128, p.n_queries - (s % p.q_tiles) * 128) - half * 64;
        if (tile_there && columns > 0) {
          const float4* l4 = reinterpret_cast<const float4*>(lse_ring + st * 128 + half * 64);
          uint64_t acc[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
#pragma unroll
          for (int ch = 0; ch < 2; ++ch) {
            if (ch * 32 >= columns) break;
            uint32_t v[32];
            tmem_ld32(s_addr + buf * 256 + ch * 32, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float4 l = l4[ch * 8 + i];
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint64_t x2 = fma_f32x2(pack_f32x2(__uint_as_float(v[4 * i + 2 * k]), __uint_as_float(v[4 * i + 2 * k + 1])), c2,
                                              k ? pack_f32x2(l.z, l.w) : pack_f32x2(l.x, l.y));
                float x0, x1, e0, e1;
                unpack_f32x2(x2, x0, x1);
                if (k == 1 && (i & POBS_POLY_MASK) == POBS_POLY_MASK) {
                  // held within the exponents of a float (2^128 is infinity); a NaN, which that would drop, comes back through the product with zero
                  ex2_poly5_pair(pack_f32x2(fminf(fmaxf(x0, -126.f), 128.f), fminf(fmaxf(x1, -126.f), 128.f)), e0, e1);
                  acc[k] = add_f32x2(acc[k], fma_f32x2(x2, pack_f32x2(0.f, 0.f), pack_f32x2(e0, e1)));
                } else {
                  e0 = ex2_approx(x0);
                  e1 = ex2_approx(x1);
                  acc[k] = add_f32x2(acc[k], pack_f32x2(e0, e1));
                }
              }
            }
          }
          float a0, a1;
          unpack_f32x2(add_f32x2(acc[0], acc[1]), a0, a1);
          sum += a0 + a1;
        }
        tc_fence_before_sync();
        __threadfence_block();  // the log-sum-exps have been read, not only asked for, when their slot is given back
        __syncwarp();
        mbar_arrive_if(&bar_s_free[buf], lane == 0);
        mbar_arrive_if(&bar_l_free[st], lane == 0);
      }
      // the two halves of a token's columns become one (these barriers are met whatever the waits gave)
      if (half) other_half[t * 128 + r] = sum;
      asm volatile("bar.sync 1, 512;" ::: "memory");
      if (!half && ok) {
        sum += other_half[t * 128 + r];
        if (w.slot >= 0) {
          p.part[static_cast<size_t>(w.slot) * 256 + t * 128 + r] = sum;
        } else if (token < p.len.n[w.head]) {
          float* dst = p.c.weights + static_cast<size_t>(w.head) * p.c.cap + token;
          *dst = (p.decay == 0.f ? 0.f : p.decay * *dst) + sum;
        }
      }
      asm volatile("bar.sync 1, 512;" ::: "memory");
    }
  }
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// Joins the sums of pairs of tiles that were cut; blocks are dealt by boundary between two shares as in packed_merge_kernel.
__global__ void __launch_bounds__(256) packed_observe_merge_kernel(const __grid_constant__ PackedObserveParams p) {
  pdl_launch_dependents();
  const int boundary = 1 + blockIdx.x;
  const int64_t total = p.line_first[p.c.n_kv], at = share_begin(boundary, total, p.n_cta);
  int head = 0;
  while (p.line_first[head + 1] <= at) ++head;
  const int steps = p.group * p.q_tiles;
  const int pair = static_cast<int>((at - p.line_first[head]) / steps);
  const int64_t first = p.line_first[head] + static_cast<int64_t>(pair) * steps;
  const int b0 = share_owner(first, total, p.n_cta), b1 = share_owner(first + steps - 1, total, p.n_cta);
  const int token = pair * 256 + threadIdx.x;
  pdl_wait();
  if (at == first || boundary != b0 + 1 || token >= p.len.n[head] || *reinterpret_cast<volatile int32_t*>(p.c.status) != 0) return;
  float sum = p.part[static_cast<size_t>(2 * b0 + 1) * 256 + threadIdx.x];
  for (int b = b0 + 1; b <= b1; ++b) sum += p.part[static_cast<size_t>(2 * b) * 256 + threadIdx.x];
  float* dst = p.c.weights + static_cast<size_t>(head) * p.c.cap + token;
  *dst = (p.decay == 0.f ? 0.f : p.decay * *dst) + sum;
}

// weight *= decay, for calls without queries.
__global__ void __launch_bounds__(256) packed_decay_kernel(const __grid_constant__ PackedObserveParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int token = blockIdx.x * 256 + threadIdx.x;
  if (token >= p.len.n[blockIdx.y]) return;
  float* dst = p.c.weights + static_cast<size_t>(blockIdx.y) * p.c.cap + token;
  *dst = p.decay == 0.f ? 0.f : p.decay * *dst;
}

}  // namespace hc
