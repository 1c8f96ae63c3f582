// Attention of many query rows over a packed cache, on tcgen05 tensor cores.
//
// The plan is the one of attn_kernel.cuh - a work item is up to two 128-row query tiles of one key/value head over a range of 128-token
// tiles; S = Q K^T and O += P V with S, P and O in tensor memory, one thread per query row for the softmax, one issuing
// warp - with the tile loads replaced by four warps that turn codes into operands:
//   - codes and scales arrive in shared memory by bulk copies, up to three tiles ahead; the warps convert them to fp16 (exact) and
//     write them into a ring slot in the layout that the products read (128-byte swizzle).  (Fetched into registers instead, a tile
//     took 1600 clk to convert: the fence behind its stores also waits for the loads that are under way for the next.)
//   - all operands are fp16: rows of Q are brought to a common power of two first (exact but for elements below 2^-28 of
//     their row's largest), P keeps 11 bits, so the row sum needs no rounding of its own to match;
//   - 56 / 72 / 192 / 192 registers for the issuing, converting and the two softmax warpgroups.
// Rows of a key/value head: row r is token r / group, query head head * group + r % group, so shared heads fill the tiles.
//
// The steps (one tile for both query tiles) of all items are laid end to end and every CTA, one per SM, takes an equal share; an
// item that is cut leaves partial results that packed_merge_kernel joins.  No lists: every role finds its items by division.
// The packed streams are 3.6 times smaller than bf16, so they share L2 where bf16 streams had to be taken in turn.
//
// What bounds it: a tile's softmax (1700 clk alone on its schedulers, 2000 beside the other tile's) and its products (1024, and 350 until
// their results are seen) follow one another; two tiles overlap to 3700 clk a step.  4680 queries x 32760 tokens, 12 heads of 128: 740 us,
// 1270 TFLOP/s, and 850 for seconds on end, at the power cap; 10800 x 75600: 4.37 ms.  At d = 64, 16 heads, 4680 x 32760 take 917 us, 2.4 times
// their products: what bounds them there is not known.  (Stores to spilled registers: 40 bytes a thread at d = 128, 88 at d = 64.)
#pragma once
#include "packed_format.cuh"

namespace hc {

struct PackedAttnParams {
  PackedView c;
  const __nv_bfloat16* q;  // [n_queries][n_kv * group][d]
  __nv_bfloat16* out;
  float* lse;              // [n_kv * group][n_queries] or null
  float* part_o;           // [2 * n_cta][256][d] unnormalised; slot 2b: CTA b's first item, which began elsewhere; 2b + 1: its last, which ends elsewhere
  float2* part_ml;         // [2 * n_cta][256]: reference (log2 domain) and sum
  int32_t n_queries, group, n_rows, n_pairs;  // n_rows = n_queries * group, n_pairs = ceil(n_rows / 256)
  int32_t n_cta;
  float scale_log2e;
  int64_t line_first[PACK_MAX_HEADS + 1];     // steps of the heads before h: n_pairs times their tiles
  HeadCounts len;
};

struct PackedItem {
  int32_t head, pair, tile_begin, tile_end, tiles, slot;  // slot < 0: the whole range, final
};

// The item that starts at step x of the line, and ends at `hi` at the latest; x moves behind it.
__host__ __device__ inline PackedItem packed_item(const PackedAttnParams& p, int cta, int64_t& x, int64_t hi, int& head) {
  while (p.line_first[head + 1] <= x) ++head;
  PackedItem w;
  w.head = head;
  w.tiles = (p.len.n[head] + PACK_TILE - 1) / PACK_TILE;
  const int64_t in_head = x - p.line_first[head];
  w.pair = static_cast<int32_t>(in_head / w.tiles);
  w.tile_begin = static_cast<int32_t>(in_head - static_cast<int64_t>(w.pair) * w.tiles);
  const int64_t end = w.tile_begin + (hi - x);
  w.tile_end = end < w.tiles ? static_cast<int32_t>(end) : w.tiles;
  x += w.tile_end - w.tile_begin;
  w.slot = w.tile_begin > 0 ? 2 * cta : w.tile_end < w.tiles ? 2 * cta + 1 : -1;
  return w;
}

constexpr int PATTN_THREADS = 512;  // warp 0: MMA, 1: loads, 2-3: idle, 4-7: conversion, 8-11 / 12-15: softmax of query tile 0 / 1
constexpr int PATTN_REGS_LAUNCH = 128, PATTN_REGS_ISSUE = 56, PATTN_REGS_CONVERT = 72, PATTN_REGS_SOFTMAX = 192;
static_assert(PATTN_REGS_ISSUE + PATTN_REGS_CONVERT + 2 * PATTN_REGS_SOFTMAX <= 4 * PATTN_REGS_LAUNCH, "the block cannot take more registers than it was launched with");
constexpr int PATTN_SLOTS = 4;       // ring of converted K and V tiles, K0 V0 K1 V1 ...
constexpr int PATTN_CODE_SLOTS = 3;  // and of their codes on the way in
constexpr float P_MOST = 32768.f;    // of a tile's sum of exponentials without a new reference: each then fits fp16, whose largest is 65504

// 2^f on [-1/2, 1/2]: of the polynomials with value 1 at 0 (whole powers come out exact, 2^128 as infinity) the one of least largest
// relative error (Lawson's iteration on 4001 Chebyshev points), coefficients rounded to fp32
constexpr float EX2_C0 = 1.f, EX2_C1 = 0.693147004f, EX2_C2 = 0.240222424f, EX2_C3 = 0.0555073358f, EX2_C4 = 0.00967151299f, EX2_C5 = 0.00132647273f;

template <int D>
struct PackedAttnSmem {
  static constexpr int BLOCK_BYTES = 128 * 128;  // [128 rows][64 fp16], 128-byte swizzle
  static constexpr int TILE_BYTES = (D / 64) * BLOCK_BYTES;
  static constexpr int KV_OFF = 2 * TILE_BYTES;
  static constexpr int CODE_OFF = KV_OFF + PATTN_SLOTS * TILE_BYTES;
  static constexpr int CODE_BYTES = PACK_TILE * (D / 2 + D / PACK_GROUP);  // codes, then scales
  static constexpr int DYN_BYTES = CODE_OFF + PATTN_CODE_SLOTS * CODE_BYTES + 1024;
};

// 2^x for a packed pair on the FMA pipe: x = n + f with |f| <= 1/2, a polynomial of degree five for 2^f (its relative error, 2e-7, is
// that of the special-function unit), n added to the exponent.  Inputs at least -126.
__device__ __forceinline__ void ex2_poly5_pair(uint64_t x2, float& e_lo, float& e_hi) {
  const uint64_t magic = pack_f32x2(12582912.f, 12582912.f), neg_magic = pack_f32x2(-12582912.f, -12582912.f), neg_one = pack_f32x2(-1.f, -1.f);
  const uint64_t t2 = add_f32x2(x2, magic);
  const uint64_t f2 = fma_f32x2(add_f32x2(t2, neg_magic), neg_one, x2);
  uint64_t p2 = fma_f32x2(f2, pack_f32x2(EX2_C5, EX2_C5), pack_f32x2(EX2_C4, EX2_C4));
  p2 = fma_f32x2(p2, f2, pack_f32x2(EX2_C3, EX2_C3));
  p2 = fma_f32x2(p2, f2, pack_f32x2(EX2_C2, EX2_C2));
  p2 = fma_f32x2(p2, f2, pack_f32x2(EX2_C1, EX2_C1));
  p2 = fma_f32x2(p2, f2, pack_f32x2(EX2_C0, EX2_C0));
  float t_lo, t_hi, p_lo, p_hi;
  unpack_f32x2(t2, t_lo, t_hi);
  unpack_f32x2(p2, p_lo, p_hi);
  e_lo = __uint_as_float(__float_as_uint(p_lo) + (__float_as_uint(t_lo) << 23));
  e_hi = __uint_as_float(__float_as_uint(p_hi) + (__float_as_uint(t_hi) << 23));
}

template <int D>
__global__ void __launch_bounds__(PATTN_THREADS, 1) packed_attn_kernel(const __grid_constant__ PackedAttnParams p) {
  using SM = PackedAttnSmem<D>;
  constexpr int QK_STEPS = D / 16;
  // Pairs of exponentials whose index has these bits set take the polynomial: an eighth at d = 128 (a quarter 746 us for a 30 x 52 block, an
  // eighth 729, a sixteenth 727: the last two are level), a quarter at d = 64, where the products take half the time (935 us, 970, 980 for 16 heads).
  constexpr int POLY = D == 128 ? 7 : 3;
  constexpr uint32_t TMEM_COLS = 512;
  constexpr uint32_t S_COL = 0, O_COL = 256;  // S_t at t*128, O_t at 256 + t*128; P_t overlays the first half of S_t

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = aligned_shared<1024>(smem_raw);
  __shared__ uint64_t bar_q_full[2], bar_s_full[2], bar_p_full[2], bar_o_full[2];
  __shared__ uint64_t bar_kv_full[PATTN_SLOTS], bar_kv_free[PATTN_SLOTS], bar_c_full[PATTN_CODE_SLOTS], bar_c_free[PATTN_CODE_SLOTS];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(&bar_q_full[t], 4);
      mbar_init(&bar_s_full[t], 1);
      mbar_init(&bar_p_full[t], 4);
      mbar_init(&bar_o_full[t], 1);
    }
    for (int s = 0; s < PATTN_CODE_SLOTS; ++s) {
      mbar_init(&bar_c_full[s], 1);
      mbar_init(&bar_c_free[s], 4);
    }
    for (int s = 0; s < PATTN_SLOTS; ++s) {
      mbar_init(&bar_kv_full[s], 4);
      mbar_init(&bar_kv_free[s], 1);
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
  const int64_t x_lo = share_begin(blockIdx.x, total, p.n_cta), x_hi = share_begin(blockIdx.x + 1, total, p.n_cta);
  int64_t x = x_lo;
  int head = 0;

  if (warp < 4) {
    regs_dec<PATTN_REGS_ISSUE>();
    if (warp == 0) {
      // ---------------------------------------------------------------- MMA issuer (the whole warp, converged)
      const uint32_t elected = elect_one();
      const uint32_t idesc_s = idesc_f16_f32(128, 128, 0, 0), idesc_o = idesc_f16_f32(128, D, 0, 1);
      const uint32_t q_addr = smem_u32(smem), kv_addr = smem_u32(smem + SM::KV_OFF);
      const uint64_t q_desc = smem_desc_sw128(q_addr, 16, 1024), k_desc = smem_desc_sw128(kv_addr, 16, 1024);
      const uint64_t v_desc = smem_desc_sw128(kv_addr, SM::BLOCK_BYTES, 1024);
      uint32_t kt = 0, q_cnt[2] = {0, 0}, p_cnt[2] = {0, 0};
      bool ok = true;
      auto issue_qk = [&](int t, uint32_t st) {
        mma_block_ss<QK_STEPS>(tmem + S_COL + t * 128, q_desc + ((t * SM::TILE_BYTES) >> 4), k_desc + ((st * SM::TILE_BYTES) >> 4), idesc_s,
                               SM::BLOCK_BYTES >> 4, elected);
      };
      auto wait = [&](uint64_t* bar, uint32_t parity, int code) -> bool { return mbar_wait_warp(bar, parity, abortp, p.c.status, code); };
      while (ok && x < x_hi) {
        const PackedItem w = packed_item(p, blockIdx.x, x, x_hi, head);
        const int nt = w.tile_end - w.tile_begin;
        const int n_q = w.pair * 256 + 128 < p.n_rows ? 2 : 1;
        {
          const uint32_t st = (2 * kt) % PATTN_SLOTS, ph = ((2 * kt) / PATTN_SLOTS) & 1;
          if (!(ok = wait(&bar_kv_full[st], ph, 71))) break;
          for (int t = 0; t < n_q && ok; ++t) {
            if (!(ok = wait(&bar_q_full[t], q_cnt[t] & 1, 72))) break;
            ++q_cnt[t];
            tc_fence_after_sync();
            issue_qk(t, st);
            mma_commit(&bar_s_full[t], elected);
          }
          if (!ok) break;
          mma_commit(&bar_kv_free[st], elected);
        }
        for (int j = 0; j < nt && ok; ++j) {
          const uint32_t gv = 2 * (kt + j) + 1, gk = gv + 1;  // ring positions of V_j and K_{j+1}
          const uint32_t st = gv % PATTN_SLOTS, ph = (gv / PATTN_SLOTS) & 1, st1 = gk % PATTN_SLOTS, ph1 = (gk / PATTN_SLOTS) & 1;
          if (!(ok = wait(&bar_kv_full[st], ph, 73))) break;
          if (j + 1 < nt && !(ok = wait(&bar_kv_full[st1], ph1, 74))) break;
          for (int t = 0; t < n_q && ok; ++t) {
            const uint64_t v_at = v_desc + ((st * SM::TILE_BYTES) >> 4);
            if (!(ok = wait(&bar_p_full[t], p_cnt[t] & 1, 76))) break;
            ++p_cnt[t];
            tc_fence_after_sync();
            mma_block_ts<0, 8>(tmem + O_COL + t * 128, tmem + S_COL + t * 128, v_at, idesc_o, j > 0 ? 1u : 0u, elected);
            if (j + 1 < nt) {
              issue_qk(t, st1);
              mma_commit(&bar_s_full[t], elected);
              if (t == n_q - 1) mma_commit(&bar_kv_free[st1], elected);
            } else {
              mma_commit(&bar_o_full[t], elected);
            }
          }
          if (!ok) break;
          mma_commit(&bar_kv_free[st], elected);
        }
        kt += nt;
      }
    } else if (warp == 1 && lane == 0) {
      // ---------------------------------------------------------------- codes and scales of K and V tiles, in the order of their use
      uint32_t g = 0;
      bool ok = true;
      while (ok && x < x_hi) {
        const PackedItem w = packed_item(p, blockIdx.x, x, x_hi, head);
        size_t row = static_cast<size_t>(w.head) * p.c.cap + static_cast<size_t>(w.tile_begin) * PACK_TILE;
        for (int tile = w.tile_begin; tile < w.tile_end && ok; ++tile, row += PACK_TILE)
          for (int kv = 0; kv < 2; ++kv) {
            const uint32_t cs = g % PATTN_CODE_SLOTS;
            if (!(ok = mbar_wait(&bar_c_free[cs], ((g / PATTN_CODE_SLOTS) & 1) ^ 1, abortp, p.c.status, 81))) break;
            uint8_t* dst = smem + SM::CODE_OFF + cs * SM::CODE_BYTES;
            mbar_arrive_expect_tx(&bar_c_full[cs], SM::CODE_BYTES);
            bulk_load(dst, (kv ? p.c.v_codes : p.c.k_codes) + row * (D / 2), PACK_TILE * D / 2, &bar_c_full[cs]);
            bulk_load(dst + PACK_TILE * D / 2, (kv ? p.c.v_scales : p.c.k_scales) + row * (D / PACK_GROUP), PACK_TILE * D / PACK_GROUP, &bar_c_full[cs]);
            ++g;
          }
      }
      if (!ok) {  // the copies in flight land before the block leaves
        for (uint32_t back = 1; back <= PATTN_CODE_SLOTS && back <= g; ++back) {
          int local_abort = 0;
          mbar_wait(&bar_c_full[(g - back) % PATTN_CODE_SLOTS], ((g - back) / PATTN_CODE_SLOTS) & 1, &local_abort, p.c.status, 82);
        }
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------------ conversion
    regs_dec<PATTN_REGS_CONVERT>();
    // D / 32 lanes share a row, 16 bytes of codes each; a warp converts its 32 rows in passes.  The upper half of them takes
    // its words in another order: both halves then write to different banks (they hold the same columns of different 64-column blocks).
    constexpr int PARTS = D / 32, ROWS = 32 / PARTS, PASSES = 32 / ROWS;
    const int part = lane % PARTS;
    const bool swap = PARTS == 4 && part >= 2;
    const int row0 = (warp & 3) * 32 + lane / PARTS;
    uint32_t g = 0;
    bool ok = true;
    while (ok && x < x_hi) {
      const PackedItem w = packed_item(p, blockIdx.x, x, x_hi, head);
      const uint32_t end = g + 2 * (w.tile_end - w.tile_begin);
      for (; g != end; ++g) {
        const uint32_t cs = g % PATTN_CODE_SLOTS, st = g % PATTN_SLOTS;
        if (!(ok = mbar_wait_warp(&bar_c_full[cs], (g / PATTN_CODE_SLOTS) & 1, abortp, p.c.status, 77))) break;
        const uint8_t* codes = smem + SM::CODE_OFF + cs * SM::CODE_BYTES;
        if (!(ok = mbar_wait_warp(&bar_kv_free[st], ((g / PATTN_SLOTS) & 1) ^ 1, abortp, p.c.status, 80))) break;
        uint8_t* dst = smem + SM::KV_OFF + st * SM::TILE_BYTES + (part / 2) * SM::BLOCK_BYTES;
        // one pass at a time, its words fetched during the one before: unrolled, the code of all roles together ran 7 % slower
        const uint8_t* at = codes + row0 * (D / 2) + part * 16;
        const uint8_t* at_scales = codes + PACK_TILE * D / 2 + row0 * (D / PACK_GROUP) + part * 2;
        uint4 c_next = *reinterpret_cast<const uint4*>(at);
        uint32_t sc_next = *reinterpret_cast<const uint16_t*>(at_scales);
#pragma unroll 1
        for (int i = 0; i < PASSES; ++i) {
          const uint4 c = c_next;
          const uint32_t sc = sc_next;
          if (i + 1 < PASSES) {
            c_next = *reinterpret_cast<const uint4*>(at + (i + 1) * ROWS * (D / 2));
            sc_next = *reinterpret_cast<const uint16_t*>(at_scales + (i + 1) * ROWS * (D / PACK_GROUP));
          }
          const int row = row0 + i * ROWS;
          const uint32_t words[4] = {swap ? c.z : c.x, swap ? c.w : c.y, swap ? c.x : c.z, swap ? c.y : c.w};
          const uint32_t s_lo = scale_f16x2(sc, 0), s_hi = scale_f16x2(sc, 1);
          const uint32_t s2[2] = {swap ? s_hi : s_lo, swap ? s_lo : s_hi};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int chunk = (part & 1) * 4 + (k ^ (swap ? 2 : 0));  // eight elements
            uint32_t v[4];
            codes_to_f16x2(words[k], v);
            *reinterpret_cast<uint4*>(dst + sw128_offset(row, chunk)) =
                make_uint4(mul_f16x2(v[0], s2[k / 2]), mul_f16x2(v[1], s2[k / 2]), mul_f16x2(v[2], s2[k / 2]), mul_f16x2(v[3], s2[k / 2]));
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        mbar_arrive_if(&bar_kv_full[st], lane == 0);
        // Only now, when every loaded word has been used: an arrival right behind the loads let the next copy in before they were done.
        mbar_arrive_if(&bar_c_free[cs], lane == 0);
      }
    }
  } else {
    // ------------------------------------------------------------------ softmax + epilogue: one thread per query row
    regs_inc<PATTN_REGS_SOFTMAX>();
    const int t = (warp - 8) >> 2;
    const int r = ((warp & 3) << 5) | lane;  // row inside the tile == TMEM lane
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) << 5) << 16;
    const uint32_t s_addr = tmem + lane_off + S_COL + t * 128, o_addr = tmem + lane_off + O_COL + t * 128;
    uint8_t* sq = smem + t * SM::TILE_BYTES;
    const int row0 = r & ~31;
    const int heads = p.c.n_kv * p.group;
    uint32_t s_cnt = 0, o_cnt = 0;
    bool ok = true;
    while (ok && x < x_hi) {
      const PackedItem w = packed_item(p, blockIdx.x, x, x_hi, head);
      const int base = w.pair * 256 + t * 128;  // first row of this tile
      if (base >= p.n_rows) continue;
      const bool row_valid = base + r < p.n_rows;
      // where the row is in q and out, in units of rows
      int64_t at = 0;
      if (row_valid) {
        const int token = (base + r) / p.group;
        at = static_cast<int64_t>(token) * heads + w.head * p.group + (base + r - token * p.group);
      }
      // ---- this thread's query row, as fp16 relative to a power of two of its own, into shared memory (swizzled); invalid rows are zero
      float c;  // from logits to the log2 domain
      {
        constexpr int CH = D / 8;
        uint4 v[CH];
#pragma unroll
        for (int k = 0; k < CH; ++k) v[k] = row_valid ? *(reinterpret_cast<const uint4*>(p.q + at * D) + k) : make_uint4(0, 0, 0, 0);
        // the largest magnitude as an integer: bf16 magnitudes are ordered like their bits, NaN above infinity
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < CH; ++k)
          top = __vmaxu2(__vmaxu2(top, __vmaxu2(v[k].x & 0x7fff7fffu, v[k].y & 0x7fff7fffu)), __vmaxu2(v[k].z & 0x7fff7fffu, v[k].w & 0x7fff7fffu));
        top = max(top & 0xffffu, top >> 16);
        float f, back;
        row_factor(__uint_as_float(top << 16), f, back);
        c = logit_factor(p.scale_log2e, back);
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const uint32_t raw[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
          uint32_t y[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = pack_f16x2(__uint_as_float(raw[i] << 16) * f, __uint_as_float(raw[i] & 0xffff0000u) * f);
          *reinterpret_cast<uint4*>(sq + (k / 8) * SM::BLOCK_BYTES + sw128_offset(r, k % 8)) = make_uint4(y[0], y[1], y[2], y[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before_sync();  // orders this thread's TMEM reads of the previous item before the arrive
        __syncwarp();
        mbar_arrive_if(&bar_q_full[t], lane == 0);
      }
      float m_ref = NO_REFERENCE, l_sum = 0.f;
      bool seeking = true;  // some row of the warp has no reference yet
      for (int tile = w.tile_begin; tile < w.tile_end; ++tile) {
        const int n_valid = min(PACK_TILE, p.len.n[w.head] - tile * PACK_TILE);
        if (!(ok = mbar_wait_warp(&bar_s_full[t], s_cnt & 1, abortp, p.c.status, 78))) break;
        ++s_cnt;
        tc_fence_after_sync();
        if (n_valid < PACK_TILE) {  // the last tile of a head: the columns behind its tokens, in tensor memory and in a few instructions
#pragma unroll 1
          for (int i = n_valid; i < PACK_TILE; ++i) tmem_st1(s_addr + i, 0xff800000u);
          tmem_wait_st();
        }
        // The exponentials are taken relative to the reference as it stands, without a look for the tile's maximum: their sum shows
        // whether one of them outgrew fp16 (each is at most the sum).  Only then, and until every row of the warp has a reference of
        // its own (mostly in an item's first tile), the maximum is found, the reference moved and the tile done again; the logits
        // are still there, P is stored last.
        uint32_t pk[64];
        float tile_sum;
        for (bool look = seeking;; look = true) {
          if (look) {
            float mx = -INFINITY;
#pragma unroll 1
            for (int ch = 0; ch < 4; ++ch) {
              uint32_t v[32];
              tmem_ld32(s_addr + ch * 32, v);
              tmem_wait_ld(v);
#pragma unroll
              for (int i = 0; i < 32; i += 2) mx = max3(mx, __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
            }
            mx *= c;
            if (above_limit(mx)) c = __uint_as_float(0x7fffffffu);
            if (__any_sync(0xffffffffu, mx > m_ref + P_HEADROOM + 1.f)) {
              const float m_new = mx > m_ref + P_HEADROOM ? reference_for(mx) : m_ref;
              const float alpha = ex2_approx(m_ref - m_new);
              l_sum *= alpha;
              m_ref = m_new;
              if (tile > w.tile_begin) {
#pragma unroll 1
                for (int ch = 0; ch < D / 16; ++ch) {
                  uint32_t v[16];
                  tmem_ld16(o_addr + ch * 16, v);
                  tmem_wait_ld(v);
#pragma unroll
                  for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
                  tmem_st16(o_addr + ch * 16, v);
                }
              }
            }
            seeking = __any_sync(0xffffffffu, m_ref <= LOWEST_REFERENCE);
          }
          const uint64_t c2 = pack_f32x2(c, c), m2 = pack_f32x2(-m_ref, -m_ref);
          uint64_t sum2[2] = {pack_f32x2(0.f, 0.f), pack_f32x2(0.f, 0.f)};
          uint32_t v[2][32];
          tmem_ld32(s_addr, v[0]);
#pragma unroll
          for (int ch = 0; ch < 4; ++ch) {
            tmem_wait_ld(v[ch & 1]);
            if (ch < 3) tmem_ld32(s_addr + (ch + 1) * 32, v[(ch + 1) & 1]);  // on its way while these are worked on
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const uint64_t x2 = fma_f32x2(pack_f32x2(__uint_as_float(v[ch & 1][2 * i]), __uint_as_float(v[ch & 1][2 * i + 1])), c2, m2);
              float x0, x1, e0, e1;
              unpack_f32x2(x2, x0, x1);
              if ((i & POLY) == POLY) {
                // (held within the exponents of a float; what is too large stays far too large)
                ex2_poly5_pair(pack_f32x2(fminf(fmaxf(x0, -126.f), 126.f), fminf(fmaxf(x1, -126.f), 126.f)), e0, e1);
              } else {
                e0 = ex2_approx(x0);
                e1 = ex2_approx(x1);
              }
              pk[16 * ch + i] = pack_f16x2(e0, e1);
              sum2[i & 1] = add_f32x2(sum2[i & 1], pack_f32x2(e0, e1));
            }
          }
          float a0, a1;
          unpack_f32x2(add_f32x2(sum2[0], sum2[1]), a0, a1);
          tile_sum = a0 + a1;
          // (a row of NaNs looks every time, once)
          if (look || !__any_sync(0xffffffffu, !(tile_sum <= P_MOST))) break;
        }
#pragma unroll
        for (int ch = 0; ch < 4; ++ch) tmem_st16(s_addr + ch * 16, *reinterpret_cast<uint32_t(*)[16]>(&pk[16 * ch]));
        tmem_wait_st();
        tc_fence_before_sync();
        __syncwarp();
        mbar_arrive_if(&bar_p_full[t], lane == 0);
        l_sum += tile_sum;
      }
      if (!ok) break;
      if (m_ref == NO_REFERENCE) m_ref = -INFINITY;  // no logit that is a number
      // ---- epilogue
      if (!(ok = mbar_wait_warp(&bar_o_full[t], o_cnt & 1, abortp, p.c.status, 79))) break;
      ++o_cnt;
      tc_fence_after_sync();
      // The warp turns its rows through its own 32 rows of the query buffer, which the last product has finished reading, so that
      // stores cover whole lines.
      uint8_t* stg = sq + row0 * 128;
      if (w.slot < 0) {
        l_sum = final_sum(m_ref, l_sum);
        const float inv = 1.f / l_sum;  // positive, or NaN
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t v[32];
          tmem_ld32(o_addr + ch * 32, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint4 o4;
            o4.x = pack_bf16x2(__uint_as_float(v[8 * i + 0]) * inv, __uint_as_float(v[8 * i + 1]) * inv);
            o4.y = pack_bf16x2(__uint_as_float(v[8 * i + 2]) * inv, __uint_as_float(v[8 * i + 3]) * inv);
            o4.z = pack_bf16x2(__uint_as_float(v[8 * i + 4]) * inv, __uint_as_float(v[8 * i + 5]) * inv);
            o4.w = pack_bf16x2(__uint_as_float(v[8 * i + 6]) * inv, __uint_as_float(v[8 * i + 7]) * inv);
            *reinterpret_cast<uint4*>(stg + (ch >> 1) * SM::BLOCK_BYTES + lane * 128 + ((((ch & 1) * 4 + i) ^ (lane & 7)) << 4)) = o4;
          }
        }
        __syncwarp();
        constexpr int U = D / 8;
#pragma unroll 4
        for (int k = 0; k < U; ++k) {
          const int idx = k * 32 + lane, row = idx / U, u = idx % U;
          const uint4 val = *reinterpret_cast<const uint4*>(stg + (u / 8) * SM::BLOCK_BYTES + row * 128 + (((u % 8) ^ (row & 7)) << 4));
          const int64_t to = __shfl_sync(0xffffffffu, at, row);
          const bool valid = __shfl_sync(0xffffffffu, row_valid ? 1 : 0, row) != 0;
          if (valid) *reinterpret_cast<uint4*>(p.out + to * D + u * 8) = val;
        }
        if (p.lse && row_valid) {
          const int token = (base + r) / p.group;
          p.lse[static_cast<size_t>(w.head * p.group + (base + r - token * p.group)) * p.n_queries + token] = (m_ref + log2f(l_sum)) * 0.6931471805599453f;
        }
        __syncwarp();
      } else {
        float* dst = p.part_o + (static_cast<size_t>(w.slot) * 256 + t * 128 + row0) * D;
#pragma unroll 1
        for (int ch = 0; ch < D / 32; ++ch) {
          uint32_t v[32];
          tmem_ld32(o_addr + ch * 32, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<float4*>(stg + lane * 128 + ((i ^ (lane & 7)) << 4)) =
                make_float4(__uint_as_float(v[4 * i + 0]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]));
          __syncwarp();
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int idx = k * 32 + lane, row = idx >> 3, u = idx & 7;
            const float4 val = *reinterpret_cast<const float4*>(stg + row * 128 + ((u ^ (row & 7)) << 4));
            const bool valid = __shfl_sync(0xffffffffu, row_valid ? 1 : 0, row) != 0;
            if (valid) *reinterpret_cast<float4*>(dst + static_cast<size_t>(row) * D + ch * 32 + u * 4) = val;
          }
          __syncwarp();
        }
        if (row_valid) p.part_ml[static_cast<size_t>(w.slot) * 256 + t * 128 + r] = make_float2(m_ref, l_sum);
      }
    }
  }
  // ------------------------------------------------------------------ teardown
  tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// Joins the parts of the query-tile pairs that were cut.  Blocks are dealt by pair (by_pair: of the heads that hold tokens), or, where
// those are fewer, by boundary between two shares: the first boundary inside a pair stands for the pair, the others have nothing to do.  A thread takes 8 columns of a row; GROUPS of threads share
// its parts (1, 4 or 16: the more parts, the more groups), 16 / GROUPS rows per block.
template <int D, int GROUPS>
__global__ void __launch_bounds__(16 * D / 8) packed_merge_kernel(const __grid_constant__ PackedAttnParams p, bool by_pair) {
  constexpr int C = D / 8, ROWS = 16 / GROUPS, BLOCKS = 256 / ROWS;
  __shared__ float sh_o[16][D];
  __shared__ float2 sh_ml[16];
  pdl_launch_dependents();
  const int index = blockIdx.x / BLOCKS;
  const int64_t total = p.line_first[p.c.n_kv];
  int head = 0, pair = 0;
  if (by_pair) {
    int left = index / p.n_pairs;  // heads with tokens before it
    while (p.len.n[head] == 0 || left-- > 0) ++head;
    pair = index % p.n_pairs;
  } else {
    const int64_t at = share_begin(index + 1, total, p.n_cta);
    while (p.line_first[head + 1] <= at) ++head;
    pair = static_cast<int>((at - p.line_first[head]) / ((p.len.n[head] + PACK_TILE - 1) / PACK_TILE));
  }
  const int tiles = (p.len.n[head] + PACK_TILE - 1) / PACK_TILE;
  const int64_t first = p.line_first[head] + static_cast<int64_t>(pair) * tiles;
  const int b0 = share_owner(first, total, p.n_cta), n = share_owner(first + tiles - 1, total, p.n_cta) - b0 + 1;
  const int c = threadIdx.x % C, g = (threadIdx.x / C) % GROUPS, lane_row = threadIdx.x / (C * GROUPS);
  const int in_pair = (blockIdx.x % BLOCKS) * ROWS + lane_row;
  const int row = pair * 256 + in_pair;
  pdl_wait();
  if (n < 2 || (!by_pair && index != b0) || *reinterpret_cast<volatile int32_t*>(p.c.status) != 0) return;  // the same for the whole block
  float m = -INFINITY, l = 0.f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (row < p.n_rows) {
    constexpr int BATCH = 4;  // parts whose loads are all issued before the first is used
    for (int i0 = g; i0 < n; i0 += BATCH * GROUPS) {
      float2 ml[BATCH];
      float4 a[BATCH], b[BATCH];
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        const int i = min(i0 + k * GROUPS, n - 1);
        const size_t src = static_cast<size_t>(i == 0 ? 2 * b0 + 1 : 2 * (b0 + i)) * 256 + in_pair;
        ml[k] = p.part_ml[src];
        const float4* o = reinterpret_cast<const float4*>(p.part_o + src * D + c * 8);
        asm volatile("ld.global.cs.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(a[k].x), "=f"(a[k].y), "=f"(a[k].z), "=f"(a[k].w) : "l"(o));
        asm volatile("ld.global.cs.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(b[k].x), "=f"(b[k].y), "=f"(b[k].z), "=f"(b[k].w) : "l"(o + 1));
        if (i0 + k * GROUPS >= n) ml[k].x = -INFINITY;
      }
      const float m_new = fmaxf(fmaxf(m, fmaxf(ml[0].x, ml[1].x)), fmaxf(ml[2].x, ml[3].x));
      const float old = m == -INFINITY ? 0.f : ex2_approx(m - m_new);
      m = m_new;
      l *= old;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] *= old;
#pragma unroll
      for (int k = 0; k < BATCH; ++k) {
        if (i0 + k * GROUPS >= n) continue;
        const float wgt = ml[k].x == -INFINITY ? 0.f : ex2_approx(ml[k].x - m);  // (a row of NaNs has no maximum: its NaNs count, times zero)
        l += wgt * ml[k].y;
        acc[0] += wgt * a[k].x; acc[1] += wgt * a[k].y; acc[2] += wgt * a[k].z; acc[3] += wgt * a[k].w;
        acc[4] += wgt * b[k].x; acc[5] += wgt * b[k].y; acc[6] += wgt * b[k].z; acc[7] += wgt * b[k].w;
      }
    }
  }
  if (GROUPS > 1) {
    const int mine = lane_row * GROUPS + g;
#pragma unroll
    for (int i = 0; i < 8; ++i) sh_o[mine][c * 8 + i] = acc[i];
    if (c == 0) sh_ml[mine] = make_float2(m, l);
    __syncthreads();
    if (g != 0) return;
    float top = -INFINITY;
    for (int x = 0; x < GROUPS; ++x) top = fmaxf(top, sh_ml[mine + x].x);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = 0.f;
    for (int x = 0; x < GROUPS; ++x) {
      const float wgt = sh_ml[mine + x].x == -INFINITY ? 0.f : ex2_approx(sh_ml[mine + x].x - top);
      l += wgt * sh_ml[mine + x].y;
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] += wgt * sh_o[mine + x][c * 8 + i];
    }
    m = top;
  }
  if (row >= p.n_rows) return;
  l = final_sum(m, l);
  const float inv = 1.f / l;
  const int token = row / p.group, h = head * p.group + (row - token * p.group);
  uint4 o4;
  o4.x = pack_bf16x2(acc[0] * inv, acc[1] * inv);
  o4.y = pack_bf16x2(acc[2] * inv, acc[3] * inv);
  o4.z = pack_bf16x2(acc[4] * inv, acc[5] * inv);
  o4.w = pack_bf16x2(acc[6] * inv, acc[7] * inv);
  *reinterpret_cast<uint4*>(p.out + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D + c * 8) = o4;
  if (p.lse && c == 0) p.lse[static_cast<size_t>(h) * p.n_queries + token] = (m + log2f(l)) * 0.6931471805599453f;
}

// Rows of heads that hold no token: zeros, and a log-sum-exp of -inf.
template <int D>
__global__ void __launch_bounds__(256) packed_empty_kernel(const __grid_constant__ PackedAttnParams p) {
  pdl_launch_dependents();
  pdl_wait();
  const int head = blockIdx.y;
  if (p.len.n[head] != 0) return;
  const int row = blockIdx.x * (256 / (D / 8)) + threadIdx.x / (D / 8), c = threadIdx.x % (D / 8);
  if (row >= p.n_rows) return;
  const int token = row / p.group, h = head * p.group + (row - token * p.group);
  *reinterpret_cast<uint4*>(p.out + (static_cast<size_t>(token) * (p.c.n_kv * p.group) + h) * D + c * 8) = make_uint4(0, 0, 0, 0);
  if (p.lse && c == 0) p.lse[static_cast<size_t>(h) * p.n_queries + token] = -INFINITY;
}

}  // namespace hc
