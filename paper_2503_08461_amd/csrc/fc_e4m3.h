// Rows of the 8-bit pool: e4m3 codes times one power of two per row (include/fastcache.h,
// "The 8-bit pool"), their layout and conversions.
#pragma once

#include "fc_device.h"

namespace fc {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Bytes of a layer's block: codes [2][n_heads][16][D], then exponents [2][n_heads][16].
__device__ __forceinline__ size_t e4m3_block_bytes(int n_heads, int head_dim) {
  return (size_t)32 * n_heads * (head_dim + 1);
}

// the 2^e of an exponent byte
__device__ __forceinline__ float e4m3_scale(uint32_t exponent) { return __uint_as_float(exponent << 23); }

__device__ __forceinline__ uint32_t abs_bits(_Float16 x) {
  return (uint32_t)(__builtin_bit_cast(uint16_t, x) & 0x7fffu);
}

// The largest finite magnitude of a lane's eight channels, as fp16 bits.
__device__ __forceinline__ uint32_t finite_max(half8 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = abs_bits(x[i]);
    m = max(m, a < 0x7c00u ? a : 0u);
  }
  return m;
}

// ... and of the row that LPR neighbouring lanes hold
template <int LPR>
__device__ __forceinline__ uint32_t row_max_u32(uint32_t m) {
  m = max(m, from_lane_u32<0xB1>(m));
  m = max(m, from_lane_u32<0x4E>(m));
  m = max(m, from_lane_u32<0x141>(m));
  if constexpr (LPR == 16) m = max(m, from_lane_u32<0x140>(m));
  return m;
}

// e + 127 of a row whose largest finite magnitude has these fp16 bits: 1.m * 2^E gives
// e = E - 8, one more if 1.m > 1.75 (448 = 1.75 * 2^8)
__device__ __forceinline__ int e4m3_exponent(uint32_t max_bits) {
  const uint32_t f = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)max_bits));
  const int e = (int)(f >> 23) - 8 + ((f & 0x7fffffu) > 0x600000u ? 1 : 0);  // (zero: -8)
  return min(max(e, 127 - 15), 127 + 8);
}

// Codes of a lane's eight channels: nearest, ties to even (the conversion's own rounding);
// with e = 8 they stop at 240, else at 448, which no finite channel exceeds by half a step.
__device__ __forceinline__ uint2v e4m3_codes(half8 x, int exponent) {
  const float inv = __uint_as_float((uint32_t)(254 - exponent) << 23);
  const float most = exponent == 127 + 8 ? 240.f : 448.f;
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    y[i] = fminf(fmaxf((float)x[i] * inv, -most), most);
    if (abs_bits(x[i]) >= 0x7c00u) y[i] = __builtin_nanf("");
  }
  uint2v c;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w], y[4 * w + 1], 0, false);
    c[w] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * w + 2], y[4 * w + 3], v, true);
  }
  return c;
}

// Eight codes times 2^e as fp16 numbers, exactly (every such value is one).
__device__ __forceinline__ half8 e4m3_values(uint32_t lo, uint32_t hi, float scale) {
  const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false);
  const half2v b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false);
  const half2v d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace fc
