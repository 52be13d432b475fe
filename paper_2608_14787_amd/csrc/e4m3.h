// Rows and matrices in 8 bits (e4m3 codes, a scale for each block of 128 columns): what the operators share (internal to
// libsdd).
#pragma once

#include "sdd_internal.h"

namespace sdd {

constexpr int kBlock8 = 128;     // columns (of a matrix: rows too) that share a scale
constexpr int kTile8 = 16 * kBlock8;  // bytes of a stored matrix tile: 16 rows of a block
constexpr int kMaxK8 = 1 << 20, kMaxN8 = 1 << 24, kMaxM8 = 1 << 24;

// Four values already within +-448 to their nearest e4m3 codes (ties to even), value i in byte i.
__device__ inline uint32_t codes4(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// What an E8M0 byte stands for: 2^(byte - 127); 0 is fp32's subnormal 2^-127, 255 NaN.
__device__ inline float e8m0_value(uint32_t byte) {
  const uint32_t u = byte == 0 ? 0x00400000u : byte == 255 ? 0x7fc00000u : byte << 23;
  return __builtin_bit_cast(float, u);
}

// Stored matrix: codes, then from this byte on the scales as fp32 [ceil(N / 128)][ceil(K / 128)].
inline int64_t matrix_code_bytes(const sdd_e4m3_matrix* m) { return ceil_div(m->N, 16) * ceil_div(m->K, kBlock8) * kTile8; }
int check_matrix(const sdd_e4m3_matrix* m);
// A launch counts its threads in 32 bits.
int check_grid(double blocks, int threads);

}  // namespace sdd
