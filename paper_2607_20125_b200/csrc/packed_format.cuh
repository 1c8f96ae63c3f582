// The packed (4-bit) key/value cache: how a row is held, and how kernels write and read it.
//
// Per head and token a key and a value of d elements each.  16 neighbouring elements share one scale
//   s = clamp(amax / 6 rounded to four significant bits, 2^-19, 1.875 * 2^12),
// and an element x is held as sign * s * c with c the one of 0, .5, 1, 1.5, 2, 3, 4, 6 nearest to |x| / s (ties to even,
// larger values to 6).  A NaN counts as zero.  A held value has at most six significant bits and lies between 2^-23 * odd
// and 46080: bf16 and fp16 hold it exactly, so both tensor-core types read the cache without another rounding.
//   - a scale is a byte, 5 bits of exponent over 3 of mantissa, s = (1 + m / 8) * 2^(e - 19): without subnormals, so the
//     smallest scale needs no case of its own, and any byte is a finite scale;
//   - any 4-bit code is a finite number, so rows behind the last token may hold anything: their weights are zero, and
//     zero times what they hold is zero.
// d/2 + d/16 bytes per row: 72 instead of 256 at d = 128.
#pragma once
#include <cuda_fp16.h>
#include "tc05.cuh"

namespace hc {

constexpr int PACK_GROUP = 16;       // elements that share a scale
constexpr int PACK_MAX_HEADS = 64;
constexpr int PACK_TILE = 128;       // tokens of a tile; every head's capacity is a multiple of it

// Device addresses of one cache.  Planes are [n_kv][cap]: codes d/2 bytes, scales d/16 bytes, a weight of 4 bytes per row.
struct PackedView {
  uint8_t* k_codes;
  uint8_t* v_codes;
  uint8_t* k_scales;
  uint8_t* v_scales;
  float* weights;
  int32_t* status;   // raised by a kernel that gave up on a bounded wait
  int64_t cap;       // tokens per head, a multiple of PACK_TILE
  int32_t n_kv;
  int32_t head_dim;
};
struct HeadCounts {
  int32_t n[PACK_MAX_HEADS];
};

// ---- reading.  A word holds eight elements, element 2i in the low and 2i + 1 in the high half of byte i.

// The eight values of a word without their scale, as fp16 pairs (element 2i low, 2i + 1 high): one conversion per pair.
// Measured per warp: 9 clk for eight values with the product by the scale, against 16 clk for masks, shifts and a product.
__device__ __forceinline__ void codes_to_f16x2(uint32_t w, uint32_t (&o)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
      : "r"(w));
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The scale behind byte `at` (0..3) of a word of scales.
__device__ __forceinline__ float scale_value(uint32_t bytes, int at) {
  return __uint_as_float((((bytes >> (8 * at)) & 0xffu) << 20) + (108u << 23));
}
__device__ __forceinline__ uint32_t scale_f16x2(uint32_t bytes, int at) {
  const float s = scale_value(bytes, at);
  return pack_f16x2(s, s);  // exact: four significant bits, at least 2^-19
}
// Eight held values as bf16 pairs (exact).
__device__ __forceinline__ void word_to_bf16x2(uint32_t w, float s, uint32_t (&o)[4]) {
  uint32_t h[4];
  codes_to_f16x2(w, h);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    o[i] = pack_bf16x2(f.x * s, f.y * s);
  }
}

// ---- writing.  Two neighbouring lanes share a group of 16 elements, eight each.
//
// The quotient x / s decides between codes at the borders .25, .75, ... 5.  x has 8 significant bits and s has 4, so a
// quotient that is not a border differs from it by at least 2^-10; computed as a product with an approximate 1 / s it is off by less
// than 2^-19.  Rounding it to a multiple of 2^-14 therefore puts every exact tie back on its border and moves nothing across
// one: the codes are those of exact arithmetic.  The same holds for amax / 6 and the borders of four significant bits, from which
// anything else is 2^-9 of itself away: the product with a rounded 1 / 6 is rounded to 17 bits first.
// (With two correctly rounded divisions instead, packing a 45 x 80 block took 27 us.)
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t bits = (__float_as_uint(amax * (1.f / 6.f)) + 0x40u) & ~0x7fu;
  // four significant bits: round to nearest even at bit 20 (infinity stays above every finite scale), then into the range
  const uint32_t r = (bits + 0x7ffffu + ((bits >> 20) & 1u)) >> 20;  // exponent and three bits of mantissa
  return min(max(r, 108u << 3), (108u << 3) + 255u) - (108u << 3);
}
// Eight elements, as the pairs of bf16 that they came in.
__device__ __forceinline__ uint32_t pack_word(const uint32_t (&raw)[4], uint32_t scale) {
  constexpr float snap = 768.f;  // 1.5 * 2^9: sums with it are multiples of 2^-14, of quotients of either sign
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(scale_value(scale, 0)));
  const uint64_t inv2 = pack_f32x2(inv, inv), up = pack_f32x2(snap, snap), down = pack_f32x2(-snap, -snap);
  float c[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint64_t x2 = pack_f32x2(__uint_as_float(raw[i] << 16), __uint_as_float(raw[i] & 0xffff0000u));
    unpack_f32x2(add_f32x2(fma_f32x2(x2, inv2, up), down), c[2 * i], c[2 * i + 1]);
  }
  uint32_t word;
  asm("{\n\t.reg .b8 p, q, r, s;\n\tcvt.rn.satfinite.e2m1x2.f32 p, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 q, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 r, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 s, %8, %7;\n\tmov.b32 %0, {p, q, r, s};\n\t}"
      : "=r"(word)
      : "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]), "f"(c[4]), "f"(c[5]), "f"(c[6]), "f"(c[7]));
  return word;
}

// ---- what the attention kernels share

// The first multiple of ALIGN in a block's dynamic shared memory, as an offset from it: an address rounded as an integer is a generic
// one to the compiler, and every access through it takes the path of global memory (converting a tile: 1300 clk instead of 850).
template <uint32_t ALIGN>
__device__ __forceinline__ uint8_t* aligned_shared(uint8_t* raw) {
  return raw + ((ALIGN - smem_u32(raw) % ALIGN) % ALIGN);
}
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
               "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
// Probabilities are formed relative to a reference 6 below the maximum that set it and are at most 2^14 (packed_attn_kernel bounds a tile's sum
// of them instead, by P_MOST): fp16 holds them down to 2^-24, 2^-30 of the largest.
constexpr float P_HEADROOM = 6.f, P_LAG = 14.f;
// The reference of a row that has met no logit yet (or only NaNs): below all of them, and finite, so that exponentials need no case for it.
constexpr float NO_REFERENCE = -3e38f;
// From here on (log2 domain) a reference in fp32 may be further from the largest logit than its exponential can stand: a row whose largest
// logit is not within -LOGIT_LIMIT .. LOGIT_LIMIT becomes NaN.  Upwards any logit shows it.  Downwards only all of the row's logits together
// do: while none is above -LOGIT_LIMIT the reference stays at LOWEST_REFERENCE, below that of every other row, to which such tokens are
// at most 2^P_LAG; one that stands there when all parts have been joined belongs to a row of NaNs.
constexpr float LOGIT_LIMIT = 4194304.f, LOWEST_REFERENCE = -LOGIT_LIMIT - P_LAG;
__device__ __forceinline__ bool above_limit(float mx) { return mx >= LOGIT_LIMIT; }
__device__ __forceinline__ float reference_for(float mx) { return mx > -LOGIT_LIMIT ? mx - P_HEADROOM : LOWEST_REFERENCE; }
// The sum of a row whose parts have all been joined, relative to reference m.
__device__ __forceinline__ float final_sum(float m, float sum) { return m <= LOWEST_REFERENCE ? __uint_as_float(0x7fffffffu) : sum; }

// The factor that brings a query row whose largest magnitude is `amax` to magnitudes below 2^15, and its inverse: powers of two, so
// every element of a bf16 row that is not smaller than 2^-28 of the largest is exact in fp16, and the others are off by
// less than 2^-39 of it.  A row that holds an infinity or a NaN gets NaN for the inverse: all its logits are NaN.
__device__ __forceinline__ void row_factor(float amax, float& to_f16, float& back) {
  const int e = static_cast<int>(__float_as_uint(amax) >> 23);  // biased exponent; 255: not finite
  const int f = min(187, max(1, 268 - e));                      // 2^(14 - (e - 127)), at most 2^60: smaller rows have logits of zero
  to_f16 = __uint_as_float(static_cast<uint32_t>(f) << 23);
  back = (amax < INFINITY) ? 1.f / to_f16 : __uint_as_float(0x7fffffffu);
}

// From products of such a row to logits in the log2 domain.  The largest rows at the largest scales pass what fp32 holds: a product that is not
// zero is beyond the limit with the largest factor too (it is 2^-44 at least), and one that is zero stays zero.
__device__ __forceinline__ float logit_factor(float scale_log2e, float back) {
  const float c = scale_log2e * back;
  return c > 3e38f ? 3e38f : c;
}

// A line of `total` steps is cut into n equal shares: CTA b owns [share_begin(b), share_begin(b + 1)).
__host__ __device__ inline int64_t share_begin(int64_t b, int64_t total, int64_t n) { return b * total / n; }
__host__ __device__ inline int share_owner(int64_t step, int64_t total, int64_t n) { return static_cast<int>(((step + 1) * n - 1) / total); }

}  // namespace hc
