// Attention of a few query rows (at most 16 per key/value head) over a packed cache: single tokens, and shared key heads.
//
// The work is reading the cache, 9/16 byte per element, and turning four-bit codes into tensor-core operands.  The tiles of 128
// tokens of all heads are laid end to end and every CTA (one per SM) takes an equal share; whatever part of a head it meets becomes
// a partial result (running maximum, sum, unnormalised output), and packed_merge_rows_kernel joins the parts of each row.
//   - bulk copies feed a ring of tiles (codes and scales are contiguous per head), two groups of eight warps take the tiles
//     in turn, each warp 16 of a tile's tokens with a running maximum and outputs of its own;
//   - S = Q K^T and O += P V are m16n8k16 products with the query rows as the 16 rows.  A product's inner index may be
//     permuted at will, so a lane multiplies the quarter of a row that it read with one load, and for P V it reads the same
//     16 elements of two tokens and interleaves their codes before conversion: no shuffles, no transposes;
//   - operands are fp16: held values are exact in it, query rows are brought to a common power of two first (see stage_row), and
//     probabilities keep 11 bits.  tcgen05 products want 128 rows, eight times the conversions' share here.
// About 300 warp instructions per 16 tokens (K and V, d = 128) bound it from above at 85 % of the time the memory takes.
#pragma once
#include "packed_format.cuh"

namespace hc {

constexpr int ROWS_MAX = 16;
constexpr int ROWS_GROUPS = 2, ROWS_GROUP_WARPS = 8;
constexpr int ROWS_THREADS = ROWS_GROUPS * ROWS_GROUP_WARPS * 32;
struct PackedRowsParams {
  PackedView c;
  const __nv_bfloat16* q;  // [n_queries][n_kv * group][d]; row r of head h is token r / group, head h * group + r % group
  float* part_o;           // [slot][ROWS_MAX][d], slot = CTA + head
  float2* part_ml;         // [slot][ROWS_MAX]: reference (log2 domain) and sum
  __nv_bfloat16* out;      // as q
  float* lse;              // [n_kv * group][n_queries] or null
  int32_t n_queries, group, n_rows;
  int32_t n_cta;
  float scale_log2e;
  int32_t tile_first[PACK_MAX_HEADS + 1];
  HeadCounts len;
};
template <int D>
struct RowsSmem {
  static constexpr int CODES = PACK_TILE * D / 2, SCALES = PACK_TILE * D / PACK_GROUP;
  static constexpr int STAGE = 2 * (CODES + SCALES);  // K codes, V codes, K scales, V scales
  static constexpr int STAGES = D == 128 ? 6 : 12;    // even: a stage belongs to one group
  static constexpr int Q_OFF = STAGES * STAGE;        // [D / 16][32 lanes] uint4
  static constexpr int MERGE_OFF = Q_OFF + D / 16 * 512;
  static constexpr int MERGE = ROWS_GROUP_WARPS * ROWS_MAX * D * 4;
  static constexpr int DYN_BYTES = MERGE_OFF + MERGE + 128;
};

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// One warp brings query row `r` into the operand layout: component 0 / 2 of a lane's uint4 are rows 0 to 7, 1 / 3 rows 8 to 15.
template <int D>
__device__ __forceinline__ void stage_row(uint4* qs, float* row_scale, const __nv_bfloat16* q, int r, bool valid, float scale_log2e) {
  constexpr int PER = D / 32;  // consecutive elements per lane: 4 or 2
  const int lane = threadIdx.x & 31;
  uint32_t raw[PER / 2];
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) raw[i] = valid ? reinterpret_cast<const uint32_t*>(q)[lane * (PER / 2) + i] : 0u;
  float x[PER], amax = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    x[i] = __uint_as_float((i & 1) ? (raw[i / 2] & 0xffff0000u) : (raw[i / 2] << 16));
    nan |= x[i] != x[i];
    amax = fmaxf(amax, fabsf(x[i]));
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, o));
  if (__any_sync(0xffffffffu, nan)) amax = INFINITY;
  float f, back;
  row_factor(amax, f, back);
  uint32_t* words = reinterpret_cast<uint32_t*>(qs);
#pragma unroll
  for (int i = 0; i < PER / 2; ++i) {
    const int e = lane * PER + 2 * i, quarter = e / (D / 4), w = e % (D / 4), kk = w / 4, hi = (w / 2) & 1;
    words[((kk * 32) + (r & 7) * 4 + quarter) * 4 + 2 * hi + (r >> 3)] = pack_f16x2(x[2 * i] * f, x[2 * i + 1] * f);
  }
  if (lane == 0) row_scale[r] = scale_log2e * back;
}

template <int D>
__global__ void __launch_bounds__(ROWS_THREADS, 1) packed_rows_kernel(const __grid_constant__ PackedRowsParams p) {
  using SM = RowsSmem<D>;
  constexpr int KW = D / 32;  // words of a key row that a lane reads
  constexpr int W = D / 8;    // elements of a value row that a lane reads
  constexpr int NT = D / 8;   // column tiles of O
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  __shared__ uint64_t bar_full[SM::STAGES], bar_free[SM::STAGES];
  __shared__ int abort_flag;
  __shared__ float row_scale[ROWS_MAX];
  __shared__ float warp_m[2 * ROWS_GROUP_WARPS][ROWS_MAX], warp_l[2 * ROWS_GROUP_WARPS][ROWS_MAX];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int s = 0; s < SM::STAGES; ++s) {
      mbar_init(&bar_full[s], 1);
      mbar_init(&bar_free[s], ROWS_GROUP_WARPS);
    }
    fence_mbar_init();
  }
  pdl_launch_dependents();
  pdl_wait();
  if (tid == 0) abort_flag = *reinterpret_cast<volatile int32_t*>(p.c.status) != 0;
  __syncthreads();
  if (abort_flag) return;  // a kernel gave up and the host has not heard of it yet: nothing is computed
  volatile int* abortp = &abort_flag;
  // (from here on an expired wait clears `ok`; the barriers of the block are met all the same)
  __syncthreads();
  const int total = p.tile_first[p.c.n_kv];
  const int t_lo = static_cast<int>(share_begin(blockIdx.x, total, p.n_cta)), t_hi = static_cast<int>(share_begin(blockIdx.x + 1, total, p.n_cta));
  int head = 0;
  while (p.tile_first[head + 1] <= t_lo) ++head;

  // The first thread of each group loads its group's tiles: the ring's worth now, and tile i - 2 + STAGES over tile i - 2 once tile i is
  // done, when the group's other warps have mostly left tile i - 2 as well.  (A warp for the loads would cost a quarter of
  // the registers: blocks get them for four warps at a time.)
  const bool loads = (tid % (ROWS_THREADS / ROWS_GROUPS)) == 0;
  int load_head = head, loaded = tid / (ROWS_THREADS / ROWS_GROUPS);  // the group's next tile, counted from t_lo
  auto load_tile = [&]() {
    const int t = t_lo + loaded, st = loaded % SM::STAGES;
    while (p.tile_first[load_head + 1] <= t) ++load_head;
    const size_t row = static_cast<size_t>(load_head) * p.c.cap + static_cast<size_t>(t - p.tile_first[load_head]) * PACK_TILE;
    uint8_t* dst = smem + st * SM::STAGE;
    mbar_arrive_expect_tx(&bar_full[st], SM::STAGE);
    bulk_load(dst, p.c.k_codes + row * (D / 2), SM::CODES, &bar_full[st]);
    bulk_load(dst + 2 * SM::CODES, p.c.k_scales + row * (D / PACK_GROUP), SM::SCALES, &bar_full[st]);
    bulk_load(dst + SM::CODES, p.c.v_codes + row * (D / 2), SM::CODES, &bar_full[st]);
    bulk_load(dst + 2 * SM::CODES + SM::SCALES, p.c.v_scales + row * (D / PACK_GROUP), SM::SCALES, &bar_full[st]);
    loaded += ROWS_GROUPS;
  };
  if (loads)
    while (loaded < min(t_hi - t_lo, SM::STAGES)) load_tile();
  const int group = warp / ROWS_GROUP_WARPS, key0 = (warp % ROWS_GROUP_WARPS) * 16;
  const int r = lane >> 2, q = lane & 3;
  uint4* qs = reinterpret_cast<uint4*>(smem + SM::Q_OFF);
  float* merge = reinterpret_cast<float*>(smem + SM::MERGE_OFF);
  // Column c of a product's eight tokens is token c ^ ((c >> 1) & 1): neighbouring columns differ in their row's parity
  // (K: two rows of 64 bytes per 128-byte phase), and so do every other two (V).
  const int key_row = r ^ ((r >> 1) & 1);
  const int val_a = (2 * q) ^ (q & 1), val_b = (2 * q + 1) ^ (q & 1);
  bool ok = true;
  for (int t0 = t_lo; t0 < t_hi; ++head) {
    const int t1 = min(t_hi, p.tile_first[head + 1]);
    if (t1 <= t0) continue;  // a head without tokens
    {
      const int token = warp / p.group, h = head * p.group + warp % p.group;
      stage_row<D>(qs, row_scale, p.q + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D, warp, warp < p.n_rows, p.scale_log2e);
    }
    __syncthreads();
    const float c_lo = row_scale[r], c_hi = row_scale[r + 8];
    float o[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m_lo = -INFINITY, m_hi = -INFINITY, l_lo = 0.f, l_hi = 0.f;
    for (int t = t0; t < t1; ++t) {
      const int i = t - t_lo;
      if ((i & 1) != group) continue;
      const int st = i % SM::STAGES;
      if (ok) ok = mbar_wait_warp(&bar_full[st], (i / SM::STAGES) & 1, abortp, p.c.status, 63);
      if (!ok) break;
      const uint8_t* kc = smem + st * SM::STAGE;
      const uint8_t* vc = kc + SM::CODES;
      const uint8_t* ks = kc + 2 * SM::CODES;
      const uint8_t* vs = ks + SM::SCALES;
      // S: two tiles of eight tokens
      float s[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
        const int row = key0 + 8 * j + key_row;
        uint32_t w[KW], scales;
        if (D == 128) {
          const uint4 v = *reinterpret_cast<const uint4*>(kc + row * (D / 2) + q * 16);
          w[0] = v.x; w[1] = v.y; w[KW - 2] = v.z; w[KW - 1] = v.w;
          scales = *reinterpret_cast<const uint16_t*>(ks + row * (D / PACK_GROUP) + q * 2);
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(kc + row * (D / 2) + q * 8);
          w[0] = v.x; w[1] = v.y;
          scales = *(ks + row * (D / PACK_GROUP) + q);
        }
#pragma unroll
        for (int g = 0; g < KW / 2; ++g) {
          const uint32_t sc = scale_f16x2(scales, g);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            uint32_t k4[4];
            codes_to_f16x2(w[2 * g + x], k4);
#pragma unroll
            for (int y = 0; y < 4; ++y) k4[y] = mul_f16x2(k4[y], sc);
            const int kk = 2 * (2 * g + x);
            const uint4 a = qs[kk * 32 + lane], b = qs[(kk + 1) * 32 + lane];
            mma_16816(s[j], a.x, a.y, a.z, a.w, k4[0], k4[1]);
            mma_16816(s[j], b.x, b.y, b.z, b.w, k4[2], k4[3]);
          }
        }
      }
      const int n_valid = p.len.n[head] - (t - p.tile_first[head]) * PACK_TILE - key0;  // of this warp's 16 tokens
      if (n_valid < 16) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (8 * j + val_a >= n_valid) s[j][0] = s[j][2] = -INFINITY;
          if (8 * j + val_b >= n_valid) s[j][1] = s[j][3] = -INFINITY;
        }
      }
      // the row's maximum over this warp's tokens; c may be NaN, never negative
      float mx_lo = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1])), mx_hi = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
      mx_lo = fmaxf(mx_lo, __shfl_xor_sync(0xffffffffu, mx_lo, 1));
      mx_hi = fmaxf(mx_hi, __shfl_xor_sync(0xffffffffu, mx_hi, 1));
      mx_lo = fmaxf(mx_lo, __shfl_xor_sync(0xffffffffu, mx_lo, 2)) * c_lo;
      mx_hi = fmaxf(mx_hi, __shfl_xor_sync(0xffffffffu, mx_hi, 2)) * c_hi;
      // the reference moves only when a maximum outgrows it; a warp without a valid token leaves it where it was
      const bool grow = mx_lo > m_lo + P_LAG || mx_hi > m_hi + P_LAG;
      if (__any_sync(0xffffffffu, grow)) {
        const float n_lo = mx_lo > m_lo + P_HEADROOM ? mx_lo - P_HEADROOM : m_lo, n_hi = mx_hi > m_hi + P_HEADROOM ? mx_hi - P_HEADROOM : m_hi;
        const float a_lo = n_lo == -INFINITY ? 1.f : ex2_approx(m_lo - n_lo), a_hi = n_hi == -INFINITY ? 1.f : ex2_approx(m_hi - n_hi);
        m_lo = n_lo;
        m_hi = n_hi;
        l_lo *= a_lo;
        l_hi *= a_hi;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          o[x][0] *= a_lo; o[x][1] *= a_lo;
          o[x][2] *= a_hi; o[x][3] *= a_hi;
        }
      }
      const float u_lo = m_lo == -INFINITY ? 0.f : m_lo, u_hi = m_hi == -INFINITY ? 0.f : m_hi;
      float e[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        e[j][0] = ex2_approx(fmaf(s[j][0], c_lo, -u_lo));
        e[j][1] = ex2_approx(fmaf(s[j][1], c_lo, -u_lo));
        e[j][2] = ex2_approx(fmaf(s[j][2], c_hi, -u_hi));
        e[j][3] = ex2_approx(fmaf(s[j][3], c_hi, -u_hi));
      }
      l_lo += (e[0][0] + e[0][1]) + (e[1][0] + e[1][1]);
      l_hi += (e[0][2] + e[0][3]) + (e[1][2] + e[1][3]);
      const uint32_t p0 = pack_f16x2(e[0][0], e[0][1]), p1 = pack_f16x2(e[0][2], e[0][3]), p2 = pack_f16x2(e[1][0], e[1][1]), p3 = pack_f16x2(e[1][2], e[1][3]);
      // O += P V: this lane's W elements of the tokens of columns 2q and 2q + 1 of both tiles
      {
        constexpr int VW = W / 8;  // words
        uint32_t a[2][VW], b[2][VW], sc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int ra = key0 + 8 * j + val_a, rb = key0 + 8 * j + val_b;
          if (D == 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(vc + ra * (D / 2) + r * 8), y = *reinterpret_cast<const uint2*>(vc + rb * (D / 2) + r * 8);
            a[j][0] = x.x; a[j][VW - 1] = x.y;
            b[j][0] = y.x; b[j][VW - 1] = y.y;
          } else {
            a[j][0] = *reinterpret_cast<const uint32_t*>(vc + ra * (D / 2) + r * 4);
            b[j][0] = *reinterpret_cast<const uint32_t*>(vc + rb * (D / 2) + r * 4);
          }
          const int g = r * W / PACK_GROUP;
          sc[j] = pack_f16x2(scale_value(vs[ra * (D / PACK_GROUP) + g], 0), scale_value(vs[rb * (D / PACK_GROUP) + g], 0));
        }
#pragma unroll
        for (int x = 0; x < VW; ++x) {
          uint32_t even[2][4], odd[2][4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            constexpr uint32_t LOW = 0x0f0f0f0fu;
            codes_to_f16x2((a[j][x] & LOW) | ((b[j][x] << 4) & ~LOW), even[j]);
            codes_to_f16x2(((a[j][x] >> 4) & LOW) | (b[j][x] & ~LOW), odd[j]);
          }
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            mma_16816(o[8 * x + 2 * y], p0, p1, p2, p3, mul_f16x2(even[0][y], sc[0]), mul_f16x2(even[1][y], sc[1]));
            mma_16816(o[8 * x + 2 * y + 1], p0, p1, p2, p3, mul_f16x2(odd[0][y], sc[0]), mul_f16x2(odd[1][y], sc[1]));
          }
        }
      }
      __syncwarp();
      mbar_arrive_if(&bar_free[st], lane == 0);
      if (loads && i >= ROWS_GROUPS && loaded < t_hi - t_lo) {
        const int done = i - ROWS_GROUPS;
        if (mbar_wait(&bar_free[done % SM::STAGES], (done / SM::STAGES) & 1, abortp, p.c.status, 61)) load_tile();
      }
      __syncwarp();
    }
    // ---- the sixteen warps' results become one: relative to the largest reference, eight warps' outputs at a time through shared memory
    l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 1);
    l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 1);
    l_lo += __shfl_xor_sync(0xffffffffu, l_lo, 2);
    l_hi += __shfl_xor_sync(0xffffffffu, l_hi, 2);
    if (q == 0) {
      warp_m[warp][r] = m_lo;
      warp_m[warp][r + 8] = m_hi;
      warp_l[warp][r] = l_lo;
      warp_l[warp][r + 8] = l_hi;
    }
    __syncthreads();
    float top_lo = -INFINITY, top_hi = -INFINITY;
#pragma unroll
    for (int x = 0; x < 2 * ROWS_GROUP_WARPS; ++x) {
      top_lo = fmaxf(top_lo, warp_m[x][r]);
      top_hi = fmaxf(top_hi, warp_m[x][r + 8]);
    }
    // (a row of NaN logits has no maximum; its NaNs count, times zero)
    const float f_lo = m_lo == -INFINITY ? 0.f : ex2_approx(m_lo - top_lo), f_hi = m_hi == -INFINITY ? 0.f : ex2_approx(m_hi - top_hi);
    const int slot = blockIdx.x + head;
    const int out_row = tid / (D / 4), out_chunk = tid % (D / 4);
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int phase = 0; phase < ROWS_GROUPS; ++phase) {
      if (group == phase) {
        float* mine = merge + (warp % ROWS_GROUP_WARPS) * ROWS_MAX * D;
#pragma unroll
        for (int half = 0; half < 2; ++half)  // rows r and r + 8
#pragma unroll
          for (int run = 0; run < 2; ++run)   // elements of columns 2q and 2q + 1
#pragma unroll
            for (int x = 0; x < W / 4; ++x) {
              const int row = r + 8 * half, chunk = (2 * q + run) * (W / 4) + x;
              const float f = half ? f_hi : f_lo;
              const int at = chunk ^ (((chunk >> 3) & 3) << 1) ^ (row & 1);
              *reinterpret_cast<float4*>(mine + row * D + at * 4) =
                  make_float4(o[4 * x][2 * half + run] * f, o[4 * x + 1][2 * half + run] * f, o[4 * x + 2][2 * half + run] * f, o[4 * x + 3][2 * half + run] * f);
            }
      }
      __syncthreads();
      if (out_row < ROWS_MAX) {
        const int at = out_chunk ^ (((out_chunk >> 3) & 3) << 1) ^ (out_row & 1);
#pragma unroll
        for (int x = 0; x < ROWS_GROUP_WARPS; ++x) {
          const float4 v = *reinterpret_cast<const float4*>(merge + (x * ROWS_MAX + out_row) * D + at * 4);
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
      }
      __syncthreads();
    }
    if (ok && out_row < p.n_rows)
      *reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(slot) * ROWS_MAX + out_row) * D + out_chunk * 4) = sum;
    if (ok && tid < p.n_rows) {
      float top = -INFINITY, l = 0.f;
      for (int x = 0; x < 2 * ROWS_GROUP_WARPS; ++x) top = fmaxf(top, warp_m[x][tid]);
      for (int x = 0; x < 2 * ROWS_GROUP_WARPS; ++x) l += (warp_m[x][tid] == -INFINITY ? 0.f : ex2_approx(warp_m[x][tid] - top)) * warp_l[x][tid];
      p.part_ml[static_cast<size_t>(slot) * ROWS_MAX + tid] = make_float2(top, l);
    }
    __syncthreads();  // the next head's rows overwrite what was read here
    t0 = t1;
  }
  if (loads && *abortp != 0) {  // the copies in flight land before the block leaves
    for (int back = loaded - ROWS_GROUPS; back >= 0 && back >= loaded - SM::STAGES; back -= ROWS_GROUPS) {
      int local_abort = 0;
      mbar_wait(&bar_full[back % SM::STAGES], (back / SM::STAGES) & 1, &local_abort, p.c.status, 62);
    }
  }
}

// Joins the parts of one row: out = sum 2^(m_i - m) O_i / sum 2^(m_i - m) l_i.  One block per row and head; D / 4 threads
// share a part's row, the parts are dealt over MERGE_GROUPS groups.  A head without tokens gives zeros and a log-sum-exp of -inf.
constexpr int MERGE_GROUPS = 8;

template <int D>
__global__ void __launch_bounds__(MERGE_GROUPS * D / 4) packed_merge_rows_kernel(const __grid_constant__ PackedRowsParams p) {
  constexpr int C = D / 4;
  __shared__ float4 sh_o[MERGE_GROUPS][C];
  __shared__ float2 sh_ml[MERGE_GROUPS];
  pdl_launch_dependents();
  const int row = blockIdx.x, head = blockIdx.y, c = threadIdx.x % C, g = threadIdx.x / C;
  const int total = p.tile_first[p.c.n_kv], first = p.tile_first[head], last = p.tile_first[head + 1] - 1;
  const int b0 = last >= first ? share_owner(first, total, p.n_cta) : 0, n = last >= first ? share_owner(last, total, p.n_cta) - b0 + 1 : 0;
  pdl_wait();
  if (*reinterpret_cast<volatile int32_t*>(p.c.status) != 0) return;  // a part is missing
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = g; i < n; i += MERGE_GROUPS) {
    const size_t at = static_cast<size_t>(b0 + i + head) * ROWS_MAX + row;
    const float2 ml = p.part_ml[at];
    const float4 v = *reinterpret_cast<const float4*>(p.part_o + at * D + c * 4);
    const float m_new = fmaxf(m, ml.x);
    const float old = m == -INFINITY ? 0.f : ex2_approx(m - m_new), w = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - m_new);
    m = m_new;
    l = l * old + ml.y * w;
    acc.x = acc.x * old + v.x * w; acc.y = acc.y * old + v.y * w; acc.z = acc.z * old + v.z * w; acc.w = acc.w * old + v.w * w;
  }
  sh_o[g][c] = acc;
  if (c == 0) sh_ml[g] = make_float2(m, l);
  __syncthreads();
  if (g != 0) return;
  float top = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < MERGE_GROUPS; ++i) top = fmaxf(top, sh_ml[i].x);
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < MERGE_GROUPS; ++i) {
    const float w = sh_ml[i].x == -INFINITY ? 0.f : ex2_approx(sh_ml[i].x - top);
    sum += w * sh_ml[i].y;
    const float4 v = sh_o[i][c];
    acc.x += w * v.x; acc.y += w * v.y; acc.z += w * v.z; acc.w += w * v.w;
  }
  const float inv = n == 0 ? 0.f : 1.f / sum;  // (with tokens the sum is positive, or NaN)
  const int token = row / p.group, h = head * p.group + row % p.group;
  *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D + c * 4) =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (p.lse && c == 0) p.lse[static_cast<size_t>(h) * p.n_queries + token] = n == 0 ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace hc
