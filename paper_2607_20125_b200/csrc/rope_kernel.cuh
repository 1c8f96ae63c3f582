// Rotary positions over several axes: pair i of a row turns by position(axis of i) * frequency(i).
//
// The angle is formed in turns, in 64-bit integers: a frequency is a fraction of a turn per position in units of 2^-64 turn, and
// position * frequency modulo 2^64 is the exact fractional turn, for positions of any size and sign.  Its upper 32 bits go
// to sincospif, so that a far position is as exact as a near one (an angle of 10^5 in fp32 is off by 4e-3).
// Bound by memory: every value is read and written once, 4 bytes together; 24480 tokens of 12 + 12 heads of 128 in 53 us, 5.7 TB/s.
// A block forms the sines and cosines of its tokens once, in shared memory, for all heads of queries and keys.  (Two or four loads under
// way per thread, with fewer blocks: 55 to 65 us.)
#pragma once
#include "tc05.cuh"

namespace hc {

constexpr int ROPE_MAX_PAIRS = 64;
struct RopeParams {
  const __nv_bfloat16* src[2];  // queries and keys: [n][heads][d], tokens src_stride elements apart; the second may be null
  __nv_bfloat16* dst[2];        // [n][heads][d]; may be the source where that is contiguous
  int64_t src_stride[2];
  int32_t heads[2];
  int32_t n;
  int32_t pairs, pairs_t, pairs_th;  // pairs that turn: [0, pairs_t) by time, up to pairs_th by height, the rest by width
  int32_t grid_w, frame_tokens;
  int64_t first_frame;
  const int32_t* positions;     // [n][3] or null: token i is at (first_frame + frame, row, column) of the grid
  uint64_t frequency[ROPE_MAX_PAIRS];  // in 2^-64 turns per position; negated for the inverse
};
constexpr int ROPE_THREADS = 256;
constexpr int ROPE_MANY_BLOCKS = 4 * 148;  // four for each SM of a B200: a value for tuning alone, any number of blocks gives the same results

// HALVES: pairs are (i, i + pairs) instead of (2i, 2i + 1).
// TOKENS per block: a power of two that leaves enough blocks (chosen by the caller).
template <int D, bool HALVES>
__global__ void __launch_bounds__(ROPE_THREADS, 8) rope_kernel(const __grid_constant__ RopeParams p, int tokens_per_block) {
  extern __shared__ float2 turn[];  // [tokens_per_block][D / 2] cosine and sine
  constexpr int PAIRS = D / 2;
  pdl_launch_dependents();
  if (p.positions) pdl_wait();  // the grid's positions are this call's own: their sines are formed while the kernel before ends
  const int t0 = blockIdx.x * tokens_per_block, nt = min(tokens_per_block, p.n - t0);
  for (int i = threadIdx.x; i < nt * PAIRS; i += ROPE_THREADS) {
    const int token = t0 + i / PAIRS, pair = i % PAIRS;
    if (pair >= p.pairs) continue;
    const int axis = pair < p.pairs_t ? 0 : pair < p.pairs_th ? 1 : 2;
    int64_t at;
    if (p.positions) {
      at = p.positions[3 * static_cast<size_t>(token) + axis];
    } else {
      const int frame = token / p.frame_tokens, in_frame = token - frame * p.frame_tokens, y = in_frame / p.grid_w;
      at = axis == 0 ? p.first_frame + frame : axis == 1 ? y : in_frame - y * p.grid_w;
    }
    const uint64_t turns = static_cast<uint64_t>(at) * p.frequency[pair];
    // half turns in [-1, 1): the upper 32 bits as a signed fraction
    const float half_turns = static_cast<float>(static_cast<int32_t>(turns >> 32)) * 0x1p-31f;
    float s, c;
    sincospif(half_turns, &s, &c);
    turn[i] = make_float2(c, s);
  }
  if (!p.positions) pdl_wait();
  __syncthreads();
  // what a thread turns at a time: 16 bytes of a row, in halves the 16 bytes of the partners too
  constexpr int CHUNKS = D / 8;
  const int turning = HALVES ? p.pairs / 8 : CHUNKS;                       // chunks (of first partners) that turn
  const int units = HALVES ? CHUNKS - p.pairs / 8 : CHUNKS;                // with the chunks behind them, which are copied
  for (int which = 0; which < 2; ++which) {
    if (!p.src[which]) continue;
    const int heads = p.heads[which];
    const int per_token = heads * units;
    for (int i = threadIdx.x; i < nt * per_token; i += ROPE_THREADS) {
      const int token = i / per_token, rest = i - token * per_token, h = rest / units, u = rest - h * units;
      const uint4* src = reinterpret_cast<const uint4*>(p.src[which] + static_cast<size_t>(t0 + token) * p.src_stride[which] + static_cast<size_t>(h) * D);
      uint4* dst = reinterpret_cast<uint4*>(p.dst[which] + (static_cast<size_t>(t0 + token) * heads + h) * D);
      const float2* cs = turn + token * PAIRS;
      if (HALVES) {
        if (u >= turning) {  // behind the rotated width
          const int c = u + turning;
          dst[c] = src[c];
          continue;
        }
        const uint4 a4 = src[u], b4 = src[u + turning];
        const uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
        uint32_t ya[4], yb[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 f0 = cs[8 * u + 2 * k], f1 = cs[8 * u + 2 * k + 1];
          const float a0 = __uint_as_float(a[k] << 16), a1 = __uint_as_float(a[k] & 0xffff0000u);
          const float b0 = __uint_as_float(b[k] << 16), b1 = __uint_as_float(b[k] & 0xffff0000u);
          ya[k] = pack_bf16x2(a0 * f0.x - b0 * f0.y, a1 * f1.x - b1 * f1.y);
          yb[k] = pack_bf16x2(a0 * f0.y + b0 * f0.x, a1 * f1.y + b1 * f1.x);
        }
        dst[u] = make_uint4(ya[0], ya[1], ya[2], ya[3]);
        dst[u + turning] = make_uint4(yb[0], yb[1], yb[2], yb[3]);
      } else {
        const uint4 a4 = src[u];
        uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int pair = 4 * u + k;
          if (pair < p.pairs) {  // what lies behind the rotated width keeps its bits
            const float2 f = cs[pair];
            const float x0 = __uint_as_float(a[k] << 16), x1 = __uint_as_float(a[k] & 0xffff0000u);
            a[k] = pack_bf16x2(x0 * f.x - x1 * f.y, x0 * f.y + x1 * f.x);
          }
        }
        dst[u] = make_uint4(a[0], a[1], a[2], a[3]);
      }
    }
  }
}

}  // namespace hc
