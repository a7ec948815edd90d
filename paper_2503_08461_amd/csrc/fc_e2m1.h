// Rows of the 4-bit pool: e2m1 codes times one power of two for every 32 channels
// (include/fastcache.h, "The 4-bit pool"), their layout and conversions.  The instructions round
// as the definition has it, for every fp16 number under every exponent that its group can have, and every
// value is its code's (tests/test_gpu_e2m1_conversions.py); a scale whose bits are 255 << 23 makes
// not-a-numbers of all codes.
#pragma once

#include <type_traits>

#include "fc_e4m3.h"

namespace fc {

typedef float float2v __attribute__((ext_vector_type(2)));

constexpr int kE2m1Group = 32;        // channels that share an exponent
constexpr int kE2m1NotFinite = 255;   // the exponent byte of a group that holds an infinite channel or not a number

// Bytes of a layer's block: codes [2][n_heads][16][D / 2], then exponents [2][n_heads][16][D / 32].
__device__ __forceinline__ size_t e2m1_block_bytes(int n_heads, int head_dim) { return (size_t)17 * n_heads * head_dim; }
// ... and of its codes
__device__ __forceinline__ size_t e2m1_code_bytes(int n_heads, int head_dim) { return (size_t)16 * n_heads * head_dim; }

// The largest magnitude of a lane's eight channels, as fp16 bits (infinite, not a number: 0x7c00 and more).
__device__ __forceinline__ uint32_t largest_bits(half8 x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, abs_bits(x[i]));
  return m;
}

// The exponent byte of a group whose largest magnitude has these fp16 bits: 1.m * 2^E gives
// e = E - 2, one more if 1.m > 1.5 (6 = 1.5 * 2^2); what is over 6 * 2^13 is that.
__device__ __forceinline__ int e2m1_exponent(uint32_t max_bits) {
  if (max_bits >= 0x7c00u) return kE2m1NotFinite;
  const uint32_t f = __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)max_bits));
  const int e = (int)(f >> 23) - 2 + ((f & 0x7fffffu) > 0x400000u ? 1 : 0);  // (zero: -2)
  return min(max(e, 127 - 23), 127 + 13);
}

// Codes of a lane's eight channels, the first one lowest: nearest, ties to even, at most 6.
__device__ __forceinline__ uint32_t e2m1_codes(half8 x, int exponent) {
  if (exponent == kE2m1NotFinite) return 0;
  const float scale = e4m3_scale(exponent);
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(0u, half2v{x[0], x[1]}, scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, half2v{x[2], x[3]}, scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, half2v{x[4], x[5]}, scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, half2v{x[6], x[7]}, scale, 3);
}

// The eight channels' codes and their group's exponent byte, of the four lanes (neighbours, the
// first one's number a multiple of four) that hold a group.
__device__ __forceinline__ uint32_t e2m1_group(half8 x, int* exponent) {
  uint32_t m = largest_bits(x);
  m = max(m, from_lane_u32<0xB1>(m));
  m = max(m, from_lane_u32<0x4E>(m));
  *exponent = e2m1_exponent(m);
  return e2m1_codes(x, *exponent);
}

// Eight codes times the scale as fp16 numbers, exactly (every such value is one).
__device__ __forceinline__ half8 e2m1_values(uint32_t codes, float scale) {
  const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 0);
  const half2v b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 1);
  const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 2);
  const half2v d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, 3);
  return half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// ... as fp32 numbers
__device__ __forceinline__ void e2m1_floats(uint32_t codes, float scale, float* f) {
  const float2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const float2v b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  const float2v c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
  const float2v d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  f[0] = a[0];
  f[1] = a[1];
  f[2] = b[0];
  f[3] = b[1];
  f[4] = c[0];
  f[5] = c[1];
  f[6] = d[0];
  f[7] = d[1];
}

// One lane's eight channels (piece: which) of a row on its way into a layer's blocks, whatever holds
// them there.  rh: K's heads, then V's; the row's other channels are with the lanes around this one, in order.
template <int D, int kFormat>
__device__ __forceinline__ void write_piece(void* layer, int blk, int n_heads, int rh, int slot, int piece, half8 x) {
  const size_t row = (size_t)rh * 16 + slot;
  if constexpr (kFormat == ROWS_E4M3) {
    uint8_t* block = static_cast<uint8_t*>(layer) + (size_t)blk * e4m3_block_bytes(n_heads, D);
    const int e = e4m3_exponent(row_max_u32<D / 8>(finite_max(x)));
    *reinterpret_cast<uint2v*>(block + row * D + piece * 8) = e4m3_codes(x, e);
    if (piece == 0) block[(size_t)2 * n_heads * 16 * D + row] = (uint8_t)e;
  } else if constexpr (kFormat == ROWS_E2M1) {
    uint8_t* block = static_cast<uint8_t*>(layer) + (size_t)blk * e2m1_block_bytes(n_heads, D);
    int e;
    const uint32_t codes = e2m1_group(x, &e);
    *reinterpret_cast<uint32_t*>(block + row * (D / 2) + piece * 4) = codes;
    if (piece % 4 == 0) block[e2m1_code_bytes(n_heads, D) + row * (D / 32) + piece / 4] = (uint8_t)e;
  } else {
    _Float16* block = static_cast<_Float16*>(layer) + (size_t)blk * 2 * n_heads * 16 * D;
    store_half8(block + row * D + piece * 8, x);
  }
}

// f(head size, row format), both as types
template <typename F>
void with_row_format(int head_dim, int format, F f) {
  auto with = [&](auto dim) {
    if (format == ROWS_E4M3)
      f(dim, std::integral_constant<int, ROWS_E4M3>());
    else if (format == ROWS_E2M1)
      f(dim, std::integral_constant<int, ROWS_E2M1>());
    else
      f(dim, std::integral_constant<int, ROWS_F16>());
  };
  if (head_dim == 128)
    with(std::integral_constant<int, 128>());
  else
    with(std::integral_constant<int, 64>());
}

}  // namespace fc
