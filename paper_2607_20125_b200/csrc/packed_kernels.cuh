// Writing rows into a packed cache and reading them back.
#pragma once
#include "packed_format.cuh"

namespace hc {

// A thread takes eight elements: 16 bytes of bf16, 4 of codes; two neighbours share a scale.  D / 8 threads share a row and a block takes
// PACK_UNROLL times PACK_THREADS * 8 / D consecutive tokens of one head: the rows it writes are one contiguous range of
// codes, and every load and store of a warp covers whole 32-byte sectors (with 16 elements per thread, two 16-byte accesses half a
// sector each, reading a 45 x 80 block back took 20 us instead of 13).  Reading back is bound by memory, packing by its integer work: a 45 x 80
// block takes 17.5 us and 11.6.
struct PackParams {
  PackedView c;
  const __nv_bfloat16* k;  // [n][n_kv][d], rows of tokens `stride` elements apart
  const __nv_bfloat16* v;
  int64_t stride;
  int32_t n;
  HeadCounts first;        // the slot of the first new token, per head
};
constexpr int PACK_THREADS = 256, PACK_UNROLL = 4;
__host__ __device__ constexpr int pack_block_tokens(int d) { return PACK_UNROLL * PACK_THREADS * 8 / d; }

template <int D>
__global__ void __launch_bounds__(PACK_THREADS) pack_rows_kernel(const __grid_constant__ PackParams p) {
  constexpr int U = D / 8, STEP = PACK_THREADS / U;
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int u = threadIdx.x % U;
  const int token0 = blockIdx.x * pack_block_tokens(D) + threadIdx.x / U;
  const __nv_bfloat16* src = (is_v ? p.v : p.k) + static_cast<size_t>(h) * D + 8 * u;
  uint4 raw[PACK_UNROLL];
#pragma unroll
  for (int i = 0; i < PACK_UNROLL; ++i) {
    const int token = token0 + i * STEP;
    raw[i] = make_uint4(0, 0, 0, 0);
    if (token < p.n) raw[i] = *reinterpret_cast<const uint4*>(src + static_cast<size_t>(token) * p.stride);
  }
#pragma unroll
  for (int i = 0; i < PACK_UNROLL; ++i) {
    uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
    // magnitudes of bf16 are ordered like their bits, a NaN above infinity
    auto largest = [&]() {
      uint32_t top = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) top = __vmaxu2(top, w[k] & 0x7fff7fffu);
      return max(top & 0xffffu, top >> 16);
    };
    uint32_t top = largest();
    if (top > 0x7f80u) {  // a NaN counts as zero
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] &= __vcmpleu2(w[k] & 0x7fff7fffu, 0x7f807f80u);
      top = largest();
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t scale = scale_byte(__uint_as_float(top << 16));
    const uint32_t word = pack_word(w, scale);
    const int token = token0 + i * STEP;
    if (token >= p.n) continue;
    const size_t row = static_cast<size_t>(h) * p.c.cap + p.first.n[h] + token;
    reinterpret_cast<uint32_t*>(is_v ? p.c.v_codes : p.c.k_codes)[row * U + u] = word;
    if (!(u & 1)) (is_v ? p.c.v_scales : p.c.k_scales)[row * (U / 2) + u / 2] = static_cast<uint8_t>(scale);
    if (!is_v && u == 1) p.c.weights[row] = 0.f;
  }
}

// The held values as bf16, [n_kv][n][d]: rows of tokens that a head does not have are left as they are.
struct UnpackParams {
  PackedView c;
  __nv_bfloat16* k;  // either may be null
  __nv_bfloat16* v;
  int32_t n;         // rows of an output per head
  int32_t first;     // the first token
  HeadCounts len;
};

template <int D>
__global__ void __launch_bounds__(PACK_THREADS) unpack_rows_kernel(const __grid_constant__ UnpackParams p) {
  constexpr int U = D / 8, STEP = PACK_THREADS / U;
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  __nv_bfloat16* out = is_v ? p.v : p.k;
  if (!out) return;
  const int u = threadIdx.x % U;
  const int token0 = blockIdx.x * pack_block_tokens(D) + threadIdx.x / U, n = min(p.n, p.len.n[h] - p.first);
  const size_t row0 = static_cast<size_t>(h) * p.c.cap + p.first;
  const uint32_t* codes = reinterpret_cast<const uint32_t*>(is_v ? p.c.v_codes : p.c.k_codes);
  const uint8_t* scales = is_v ? p.c.v_scales : p.c.k_scales;
  uint32_t w[PACK_UNROLL], s[PACK_UNROLL];
#pragma unroll
  for (int i = 0; i < PACK_UNROLL; ++i) {
    const int token = token0 + i * STEP;
    if (token < n) {
      w[i] = codes[(row0 + token) * U + u];
      s[i] = scales[(row0 + token) * (U / 2) + u / 2];
    }
  }
#pragma unroll
  for (int i = 0; i < PACK_UNROLL; ++i) {
    const int token = token0 + i * STEP;
    if (token >= n) continue;
    uint32_t v[4];
    word_to_bf16x2(w[i], scale_value(s[i], 0), v);
    *reinterpret_cast<uint4*>(out + (static_cast<size_t>(h) * p.n + token) * D + 8 * u) = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

}  // namespace hc
