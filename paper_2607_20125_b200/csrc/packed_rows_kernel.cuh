// Attention of a few query rows (at most 16 per key/value head) over a packed cache: single tokens, and shared key heads.
//
// The work is reading the cache, 9/16 byte per element, and turning four-bit codes into tensor-core operands.  The tiles of 128
// tokens of all heads are laid end to end and every CTA (one per SM) takes an equal share; whatever part of a head it meets becomes
// a partial result (running maximum, sum, unnormalised output), and packed_merge_rows_kernel joins the parts of each row.
//   - two groups of eight warps take the tiles in turn, each warp 16 of a tile's tokens with a running maximum and outputs of its
//     own.  Codes and scales go straight into the registers that their conversion reads, which are filled for the next tile as soon as
//     they have been used; with a ring of bulk copies in shared memory, whatever its depth, one query took 21.3 us instead of 18.1 over 32760 tokens and 59
//     instead of 52 over 131072, 16 queries 28.0 instead of 26.7 and 76 instead of 83;
//   - S^T = K Q^T and O^T += V^T P^T are m16n8k16 products, tokens (then value elements) on the 16 rows and eight queries on
//     the columns: with the queries on the 16 rows there were twice the products.  A product's inner index may be permuted at will, so a
//     lane multiplies the quarter of a row that it read with one load, and for V it reads the same 16 elements of two
//     tokens and interleaves their codes before conversion; P is turned around by movmatrix;
//   - the maximum is only looked for, across lanes, when some logit outgrows the reference;
//   - operands are fp16: held values are exact in it, query rows are brought to a common power of two first (see row_factor), and
//     probabilities keep 11 bits.  tcgen05 products want 128 rows, eight times the conversions' share here.
// One query, 12 heads of 128: 18.1 us for 32760 tokens (3.1 TB/s), 52 for 131072 (4.3 TB/s).  Latency bounds it, between the loads of a tile, their
// conversion and the products: the integer pipe, the busiest, is at 51 %, memory at 45 %.  8 us of the first are launches, first loads and the merge.
#pragma once
#include "packed_format.cuh"

namespace hc {

constexpr int ROWS_MAX = 16;
constexpr int ROWS_GROUP_WARPS = 8;
constexpr int ROWS_GROUPS = 2;  // of warps (a third one, at 80 registers a thread, made the call for one token 9 % slower)
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

// 8 x 8 values of 16 bits, two of a row per lane: the same with rows and columns exchanged.
__device__ __forceinline__ uint32_t turn_8x8(uint32_t v) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

template <int D>
struct RowsSmem {
  static constexpr int Q_BYTES = D / 16 * 512;  // [D / 16][2 query tiles][32 lanes] uint2
  static constexpr int DYN_BYTES = Q_BYTES + ROWS_GROUPS * ROWS_GROUP_WARPS * 8 * D * 4;  // and every warp's outputs
};

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// One warp brings query row `r` into the operand layout: the lane of row r % 8 and quarter c holds, for each product, four elements
// of that quarter.
template <int D>
__device__ __forceinline__ void stage_row(uint2* qs, float* row_scale, const __nv_bfloat16* q, int r, bool valid, float scale_log2e) {
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
    words[((kk * 2 + (r >> 3)) * 32 + (r & 7) * 4 + quarter) * 2 + hi] = pack_f16x2(x[2 * i] * f, x[2 * i + 1] * f);
  }
  if (lane == 0) row_scale[r] = logit_factor(scale_log2e, back);
}

// NQ: tiles of eight query rows
template <int D, int NQ>
__global__ void __launch_bounds__(ROWS_THREADS, 1) packed_rows_kernel(const __grid_constant__ PackedRowsParams p) {
  constexpr int GROUPS = ROWS_GROUPS, WARPS = GROUPS * ROWS_GROUP_WARPS;
  constexpr int KW = D / 32;  // words of a key row that a lane reads
  constexpr int W = D / 8;    // elements of a value row that a lane reads
  constexpr int NT = D / 16;  // row tiles of O^T
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float row_scale[ROWS_MAX];
  __shared__ float warp_m[WARPS][ROWS_MAX], warp_l[WARPS][ROWS_MAX];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int total = p.tile_first[p.c.n_kv];
  const int t_lo = static_cast<int>(share_begin(blockIdx.x, total, p.n_cta)), t_hi = static_cast<int>(share_begin(blockIdx.x + 1, total, p.n_cta));
  int head = 0;
  while (p.tile_first[head + 1] <= t_lo) ++head;
  const int group = warp / ROWS_GROUP_WARPS, key0 = (warp % ROWS_GROUP_WARPS) * 16;
  const int r = lane >> 2, q = lane & 3;
  uint2* qs = reinterpret_cast<uint2*>(smem);
  float* merge = reinterpret_cast<float*>(smem + RowsSmem<D>::Q_BYTES);
  // What a lane reads of a tile: a quarter of the keys of two tokens, 16 elements of the values of four; the rows of S^T are the
  // tokens key0 + r and key0 + 8 + r, and P^T wants those of rows 2q and 2q + 1 of both halves.
  uint32_t kw[2][KW], k_scales[2];
  constexpr int VW = W / 8;  // words
  uint32_t va[2][VW], vb[2][VW], v_scales[2][2];
  auto fetch_k = [&](int h, int tile) {
    const size_t row0 = static_cast<size_t>(h) * p.c.cap + static_cast<size_t>(tile) * PACK_TILE + key0 + r;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const size_t row = row0 + 8 * j;
      if (D == 128) {
        const uint4 v = *reinterpret_cast<const uint4*>(p.c.k_codes + row * (D / 2) + q * 16);
        kw[j][0] = v.x; kw[j][1] = v.y; kw[j][KW - 2] = v.z; kw[j][KW - 1] = v.w;
        k_scales[j] = *reinterpret_cast<const uint16_t*>(p.c.k_scales + row * (D / PACK_GROUP) + q * 2);
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p.c.k_codes + row * (D / 2) + q * 8);
        kw[j][0] = v.x; kw[j][1] = v.y;
        k_scales[j] = p.c.k_scales[row * (D / PACK_GROUP) + q];
      }
    }
  };
  auto fetch_v = [&](int h, int tile) {
    const size_t row0 = static_cast<size_t>(h) * p.c.cap + static_cast<size_t>(tile) * PACK_TILE + key0 + 2 * q;
    const int g = r * W / PACK_GROUP;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const size_t row = row0 + 8 * j;
      if (D == 128) {
        const uint2 x = *reinterpret_cast<const uint2*>(p.c.v_codes + row * (D / 2) + r * 8), y = *reinterpret_cast<const uint2*>(p.c.v_codes + (row + 1) * (D / 2) + r * 8);
        va[j][0] = x.x; va[j][VW - 1] = x.y;
        vb[j][0] = y.x; vb[j][VW - 1] = y.y;
      } else {
        va[j][0] = *reinterpret_cast<const uint32_t*>(p.c.v_codes + row * (D / 2) + r * 4);
        vb[j][0] = *reinterpret_cast<const uint32_t*>(p.c.v_codes + (row + 1) * (D / 2) + r * 4);
      }
      v_scales[j][0] = p.c.v_scales[row * (D / PACK_GROUP) + g];
      v_scales[j][1] = p.c.v_scales[(row + 1) * (D / PACK_GROUP) + g];
    }
  };
  pdl_launch_dependents();
  pdl_wait();
  int mine = group;  // this group's next tile, counted from t_lo
  for (int t0 = t_lo; t0 < t_hi; ++head) {
    const int t1 = min(t_hi, p.tile_first[head + 1]);
    if (t1 <= t0) continue;  // a head without tokens
    const int first = t_lo - p.tile_first[head];  // of this head's tiles, where `mine` is 0
    if (mine < t1 - t_lo) {
      fetch_k(head, first + mine);
      fetch_v(head, first + mine);
    }
    if (warp < 8 * NQ) {
      const int token = warp / p.group, h = head * p.group + warp % p.group;
      stage_row<D>(qs, row_scale, p.q + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D, warp, warp < p.n_rows, p.scale_log2e);
    }
    __syncthreads();
    float c[NQ][2], m[NQ][2], l[NQ][2];  // of this lane's two queries per tile: columns 2q and 2q + 1
    float o[NQ][NT][4];
#pragma unroll
    for (int z = 0; z < NQ; ++z) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        c[z][y] = row_scale[8 * z + 2 * q + y];
        m[z][y] = NO_REFERENCE;
        l[z][y] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) o[z][i][0] = o[z][i][1] = o[z][i][2] = o[z][i][3] = 0.f;
    }
    const int last_tile = p.tile_first[head + 1] - 1 - t_lo;  // of the head
    const int last_valid = p.len.n[head] - (last_tile + t_lo - p.tile_first[head]) * PACK_TILE - key0;  // of this warp's 16 tokens there
    for (; mine < t1 - t_lo; mine += GROUPS) {
      // S^T: 16 tokens
      float s[NQ][4], s_odd[NQ][4];  // two chains of products (one where registers are short)
#pragma unroll
      for (int z = 0; z < NQ; ++z)
#pragma unroll
        for (int y = 0; y < 4; ++y) s[z][y] = s_odd[z][y] = 0.f;
      {
#pragma unroll
        for (int x = 0; x < KW; ++x) {
          uint32_t a[2][4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const uint32_t sc = scale_f16x2(k_scales[j], x / 2);
            codes_to_f16x2(kw[j][x], a[j]);
#pragma unroll
            for (int y = 0; y < 4; ++y) a[j][y] = mul_f16x2(a[j][y], sc);
          }
#pragma unroll
          for (int z = 0; z < NQ; ++z) {
            const uint2 b0 = qs[(4 * x + z) * 32 + lane], b1 = qs[(4 * x + 2 + z) * 32 + lane];
            mma_16816(s[z], a[0][0], a[1][0], a[0][1], a[1][1], b0.x, b0.y);
            mma_16816(NQ == 1 ? s_odd[z] : s[z], a[0][2], a[1][2], a[0][3], a[1][3], b1.x, b1.y);
          }
        }
#pragma unroll
        for (int z = 0; z < NQ; ++z)
#pragma unroll
          for (int y = 0; y < 4; ++y) s[z][y] += NQ == 1 ? s_odd[z][y] : 0.f;
      }
      // the registers are filled for the group's next tile as soon as they have been used
      const bool more = mine + GROUPS < t1 - t_lo;
      if (more) fetch_k(head, first + mine + GROUPS);
      if (mine == last_tile) {
#pragma unroll
        for (int z = 0; z < NQ; ++z) {
          if (r >= last_valid) s[z][0] = s[z][1] = -INFINITY;
          if (8 + r >= last_valid) s[z][2] = s[z][3] = -INFINITY;
        }
      }
      // The reference moves only when some logit outgrows it (a NaN never does); tokens that are not there leave it.
      float x[NQ][4];
      bool grow = false;
#pragma unroll
      for (int z = 0; z < NQ; ++z) {
#pragma unroll
        for (int y = 0; y < 4; ++y) x[z][y] = fmaf(s[z][y], c[z][y & 1], -m[z][y & 1]);
        grow |= fmaxf(fmaxf(x[z][0], x[z][1]), fmaxf(x[z][2], x[z][3])) > P_LAG;
      }
      if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
        for (int z = 0; z < NQ; ++z)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float mx = fmaxf(s[z][y], s[z][y + 2]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
            mx *= c[z][y];
            if (above_limit(mx)) c[z][y] = __uint_as_float(0x7fffffffu);
            const float to = mx > m[z][y] + P_HEADROOM ? reference_for(mx) : m[z][y];
            const float f = ex2_approx(m[z][y] - to);
            m[z][y] = to;
            l[z][y] *= f;
#pragma unroll
            for (int x = 0; x < NT; ++x) {
              o[z][x][y] *= f;
              o[z][x][y + 2] *= f;
            }
          }
#pragma unroll
        for (int z = 0; z < NQ; ++z)
#pragma unroll
          for (int y = 0; y < 4; ++y) x[z][y] = fmaf(s[z][y], c[z][y & 1], -m[z][y & 1]);
      }
      uint32_t pt[NQ][2];  // P^T as the products want it: two tokens of one query
#pragma unroll
      for (int z = 0; z < NQ; ++z) {
        const float e0 = ex2_approx(x[z][0]), e1 = ex2_approx(x[z][1]), e2 = ex2_approx(x[z][2]), e3 = ex2_approx(x[z][3]);
        l[z][0] += e0 + e2;
        l[z][1] += e1 + e3;
        pt[z][0] = turn_8x8(pack_f16x2(e0, e1));
        pt[z][1] = turn_8x8(pack_f16x2(e2, e3));
      }
      // O^T += V^T P^T: this lane's W elements of the tokens of rows 2q and 2q + 1 of both halves
      {
        uint32_t sc[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) sc[j] = pack_f16x2(scale_value(v_scales[j][0], 0), scale_value(v_scales[j][1], 0));
#pragma unroll
        for (int x = 0; x < VW; ++x) {
          uint32_t even[2][4], odd[2][4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            constexpr uint32_t LOW = 0x0f0f0f0fu;
            codes_to_f16x2((va[j][x] & LOW) | ((vb[j][x] << 4) & ~LOW), even[j]);
            codes_to_f16x2(((va[j][x] >> 4) & LOW) | (vb[j][x] & ~LOW), odd[j]);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              even[j][y] = mul_f16x2(even[j][y], sc[j]);
              odd[j][y] = mul_f16x2(odd[j][y], sc[j]);
            }
          }
#pragma unroll
          for (int y = 0; y < 4; ++y)  // elements 8x + 2y on rows r, 8x + 2y + 1 on rows r + 8
#pragma unroll
            for (int z = 0; z < NQ; ++z) mma_16816(o[z][4 * x + y], even[0][y], odd[0][y], even[1][y], odd[1][y], pt[z][0], pt[z][1]);
        }
      }
      if (more) fetch_v(head, first + mine + GROUPS);
    }
    // ---- the warps' results become one, relative to the largest reference, through shared memory
#pragma unroll
    for (int z = 0; z < NQ; ++z)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[z][y] += __shfl_xor_sync(0xffffffffu, l[z][y], x);
        if (r == 0) {
          warp_m[warp][8 * z + 2 * q + y] = m[z][y] == NO_REFERENCE ? -INFINITY : m[z][y];
          warp_l[warp][8 * z + 2 * q + y] = l[z][y];
        }
      }
    __syncthreads();
    const int slot = blockIdx.x + head;
    if (tid < p.n_rows) {
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int x = 0; x < WARPS; ++x) top = fmaxf(top, warp_m[x][tid]);
#pragma unroll
      for (int x = 0; x < WARPS; ++x) sum += (warp_m[x][tid] == -INFINITY ? 0.f : ex2_approx(warp_m[x][tid] - top)) * warp_l[x][tid];
      p.part_ml[static_cast<size_t>(slot) * ROWS_MAX + tid] = make_float2(top, sum);
    }
#pragma unroll
    for (int z = 0; z < NQ; ++z) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int query = 2 * q + y;
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < WARPS; ++x) top = fmaxf(top, warp_m[x][8 * z + query]);
        // (a row of NaN logits has no maximum; its NaNs count, times zero)
        const float f = m[z][y] == NO_REFERENCE ? 0.f : ex2_approx(m[z][y] - top);
        float* to = merge + (warp * 8 + query) * D;
#pragma unroll
        for (int x = 0; x < W / 4; ++x)
          *reinterpret_cast<float4*>(to + ((r * (W / 4) + x) ^ q) * 4) =
              make_float4(o[z][2 * x][y] * f, o[z][2 * x][y + 2] * f, o[z][2 * x + 1][y] * f, o[z][2 * x + 1][y + 2] * f);
      }
      __syncthreads();
      const int query = tid / (D / 4), chunk = tid % (D / 4);
      if (query < 8 && 8 * z + query < p.n_rows) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int x = 0; x < WARPS; ++x) {
          const float4 v = *reinterpret_cast<const float4*>(merge + (x * 8 + query) * D + (chunk ^ (query >> 1)) * 4);
          sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
        }
        *reinterpret_cast<float4*>(p.part_o + (static_cast<size_t>(slot) * ROWS_MAX + 8 * z + query) * D + chunk * 4) = sum;
      }
      __syncthreads();  // what was read here is overwritten by the next tile of queries, or the next head's rows
    }
    t0 = t1;
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
  sum = final_sum(top, sum);
  const float inv = n == 0 ? 0.f : 1.f / sum;  // (with tokens the sum is positive, or NaN)
  const int token = row / p.group, h = head * p.group + row % p.group;
  *reinterpret_cast<uint2*>(p.out + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D + c * 4) =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
  if (p.lse && c == 0) p.lse[static_cast<size_t>(h) * p.n_queries + token] = n == 0 ? -INFINITY : (top + log2f(sum)) * 0.6931471805599453f;
}

// What up to 16 query rows per key/value head give to every token: weight = decay * weight + sum over the rows of exp(logit - lse).
// The products are those of packed_rows_kernel without the values; a row of S^T is a token and its columns the queries, so a
// token's sum is four lanes' to add and each token belongs to one warp: no parts, no second kernel.  Keys are read straight into registers, a
// tile ahead; 80 bytes per token and head at d = 128.  One query, 32760 tokens, 12 heads of 128: 9.1 us (3.4 TB/s;
// packed_observe_kernel, for which one query is as much work as 32: 32); 131072 tokens 29.5 (4.3).  Bound like packed_rows_kernel.
struct PackedObserveRowsParams {
  PackedView c;
  const __nv_bfloat16* q;
  const float* lse;  // [n_kv * group][n_queries]
  int32_t n_queries, group, n_rows;
  float scale_log2e, decay;
  HeadCounts len;
};
constexpr int OBSERVE_ROWS_THREADS = 256;

template <int D, int NQ>
__global__ void __launch_bounds__(OBSERVE_ROWS_THREADS) packed_observe_rows_kernel(const __grid_constant__ PackedObserveRowsParams p) {
  constexpr int KW = D / 32, WARPS = OBSERVE_ROWS_THREADS / 32;
  __shared__ uint2 qs[D / 16 * 2 * 32];
  __shared__ float row_scale[ROWS_MAX], row_lse[ROWS_MAX];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q = lane & 3, head = blockIdx.y;
  pdl_launch_dependents();
  pdl_wait();
  const int len = p.len.n[head], tiles = (len + PACK_TILE - 1) / PACK_TILE;
  if (static_cast<int>(blockIdx.x) >= tiles) return;
  const size_t row0 = static_cast<size_t>(head) * p.c.cap + warp * 16 + r;  // of this lane's first token in tile 0; the second is 8 rows on
  struct Keys {
    uint32_t w[2][KW], scales[2];
  };
  auto fetch = [&](Keys& k, int tile) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const size_t row = row0 + static_cast<size_t>(tile) * PACK_TILE + 8 * j;
      if (D == 128) {
        const uint4 v = *reinterpret_cast<const uint4*>(p.c.k_codes + row * (D / 2) + q * 16);
        k.w[j][0] = v.x; k.w[j][1] = v.y; k.w[j][KW - 2] = v.z; k.w[j][KW - 1] = v.w;
        k.scales[j] = *reinterpret_cast<const uint16_t*>(p.c.k_scales + row * (D / PACK_GROUP) + q * 2);
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(p.c.k_codes + row * (D / 2) + q * 8);
        k.w[j][0] = v.x; k.w[j][1] = v.y;
        k.scales[j] = p.c.k_scales[row * (D / PACK_GROUP) + q];
      }
    }
  };
  Keys next;
  fetch(next, blockIdx.x);
  for (int i = warp; i < 8 * NQ; i += WARPS) {
    const int token = i / p.group, h = head * p.group + i % p.group;
    const bool valid = i < p.n_rows;
    stage_row<D>(qs, row_scale, p.q + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D, i, valid, p.scale_log2e);
    if (lane == 0) row_lse[i] = valid ? -1.4426950408889634f * p.lse[static_cast<size_t>(h) * p.n_queries + token] : -INFINITY;
  }
  __syncthreads();
  float c[NQ][2], l[NQ][2];  // of this lane's two queries per tile: columns 2q and 2q + 1
#pragma unroll
  for (int z = 0; z < NQ; ++z)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      c[z][y] = row_scale[8 * z + 2 * q + y];
      l[z][y] = row_lse[8 * z + 2 * q + y];
    }
  for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Keys k = next;
    if (tile + static_cast<int>(gridDim.x) < tiles) fetch(next, tile + gridDim.x);
    float s[NQ][4], s_odd[NQ][4];
#pragma unroll
    for (int z = 0; z < NQ; ++z)
#pragma unroll
      for (int y = 0; y < 4; ++y) s[z][y] = s_odd[z][y] = 0.f;
#pragma unroll
    for (int x = 0; x < KW; ++x) {
      uint32_t a[2][4];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t sc = scale_f16x2(k.scales[j], x / 2);
        codes_to_f16x2(k.w[j][x], a[j]);
#pragma unroll
        for (int y = 0; y < 4; ++y) a[j][y] = mul_f16x2(a[j][y], sc);
      }
#pragma unroll
      for (int z = 0; z < NQ; ++z) {
        const uint2 b0 = qs[(4 * x + z) * 32 + lane], b1 = qs[(4 * x + 2 + z) * 32 + lane];
        mma_16816(s[z], a[0][0], a[1][0], a[0][1], a[1][1], b0.x, b0.y);
        mma_16816(s_odd[z], a[0][2], a[1][2], a[0][3], a[1][3], b1.x, b1.y);
      }
    }
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int z = 0; z < NQ; ++z)
#pragma unroll
      for (int y = 0; y < 4; ++y) sum[y / 2] += ex2_approx(fmaf(s[z][y] + s_odd[z][y], c[z][y & 1], l[z][y & 1]));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
      sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
    }
    const int token = tile * PACK_TILE + warp * 16 + r + 8 * q;  // lane q = 0 writes the first token, q = 1 the second
    if (q < 2 && token < len) {
      float* dst = p.c.weights + static_cast<size_t>(head) * p.c.cap + token;
      *dst = (p.decay == 0.f ? 0.f : p.decay * *dst) + (q ? sum[1] : sum[0]);
    }
  }
}

}  // namespace hc
