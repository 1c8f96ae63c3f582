// Writing rows into a packed cache and reading them back.
#pragma once
#include "packed_format.cuh"

namespace hc {

// One thread packs one group of 16 elements: it reads 32 bytes and writes 8 bytes of codes and a scale byte.  d/16 neighbouring
// threads share a row, a block takes PACK_ROWS(d) consecutive tokens of one head, so that the rows it writes are one contiguous
// range (64 B of codes per row at d = 128), while its reads are whole rows of 2d bytes, a token apart.  Bound by memory at
// block sizes: 2 bytes read and 0.56 written per element, once each.
struct PackParams {
  PackedView c;
  const __nv_bfloat16* k;  // [n][n_kv][d], rows of tokens `stride` elements apart
  const __nv_bfloat16* v;
  int64_t stride;
  int32_t n;
  HeadCounts first;        // the slot of the first new token, per head
};
constexpr int PACK_THREADS = 256;

template <int D>
__global__ void __launch_bounds__(PACK_THREADS) pack_rows_kernel(const __grid_constant__ PackParams p) {
  constexpr int G = D / PACK_GROUP;
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  const int g = threadIdx.x % G;
  const int token = blockIdx.x * (PACK_THREADS / G) + threadIdx.x / G;
  if (token >= p.n) return;
  const uint4* src = reinterpret_cast<const uint4*>((is_v ? p.v : p.k) + static_cast<size_t>(token) * p.stride + static_cast<size_t>(h) * D) + 2 * g;
  const uint4 q[2] = {src[0], src[1]};
  const uint32_t raw[8] = {q[0].x, q[0].y, q[0].z, q[0].w, q[1].x, q[1].y, q[1].z, q[1].w};
  float x[PACK_GROUP];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float lo = __uint_as_float(raw[i] << 16), hi = __uint_as_float(raw[i] & 0xffff0000u);
    x[2 * i] = lo != lo ? 0.f : lo;
    x[2 * i + 1] = hi != hi ? 0.f : hi;
  }
  uint32_t codes[2];
  const uint32_t scale = pack_group(x, codes);
  const size_t row = static_cast<size_t>(h) * p.c.cap + p.first.n[h] + token;
  reinterpret_cast<uint2*>(is_v ? p.c.v_codes : p.c.k_codes)[row * G + g] = make_uint2(codes[0], codes[1]);
  (is_v ? p.c.v_scales : p.c.k_scales)[row * G + g] = static_cast<uint8_t>(scale);
  if (!is_v && g == 0) p.c.weights[row] = 0.f;
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
  constexpr int G = D / PACK_GROUP;
  pdl_launch_dependents();
  pdl_wait();
  const int h = blockIdx.y;
  const bool is_v = blockIdx.z != 0;
  __nv_bfloat16* out = is_v ? p.v : p.k;
  const int g = threadIdx.x % G;
  const int token = blockIdx.x * (PACK_THREADS / G) + threadIdx.x / G;
  if (!out || token >= p.n || p.first + token >= p.len.n[h]) return;
  const size_t row = static_cast<size_t>(h) * p.c.cap + p.first + token;
  const uint2 w = reinterpret_cast<const uint2*>(is_v ? p.c.v_codes : p.c.k_codes)[row * G + g];
  const float s = scale_value((is_v ? p.c.v_scales : p.c.k_scales)[row * G + g], 0);
  uint32_t a[4], b[4];
  word_to_bf16x2(w.x, s, a);
  word_to_bf16x2(w.y, s, b);
  uint4* dst = reinterpret_cast<uint4*>(out + (static_cast<size_t>(h) * p.n + token) * D) + 2 * g;
  dst[0] = make_uint4(a[0], a[1], a[2], a[3]);
  dst[1] = make_uint4(b[0], b[1], b[2], b[3]);
}

}  // namespace hc
