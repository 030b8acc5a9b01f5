// rowquant.h -- the arithmetic of int8 rows with one scale a row, shared by
// fgq_quantize_rows (rowquant.hip) and the products that quantize their own
// rows (i8few.hip).
#pragma once

#include "fgq_internal.h"

namespace fgq {

__device__ inline uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

__device__ inline uint32_t wave_max(uint32_t m) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), off)));
  return m;
}

struct RowScale {
  float scale, r;  // r = 127 / a, or 0 for a row of zeros or with a value that is not finite
};

// m: the largest abs_bits of the row.  Below 2^-120 (127 / a would overflow)
// a row counts as zeros.
__device__ inline RowScale row_scale(uint32_t m) {
  if (m >= 0x7F800000u) return RowScale{__uint_as_float(0x7FC00000u), 0.0f};
  const float a = __uint_as_float(m);
  if (a < 0x1p-120f) return RowScale{1.0f, 0.0f};
  return RowScale{a / 127.0f, 127.0f / a};
}

// Code of x: rint(x * r).  Adding 1.5 * 2^23 rounds to even at the unit and
// leaves the code in the sum's low byte.  With r = 0 the code is 0 for every
// x (the product of a NaN or infinity is masked out).
__device__ inline uint32_t row_code(float x, float r) {
#pragma clang fp contract(off)
  const float p = x * r;
  return __float_as_uint(p + 12582912.0f);
}
__device__ inline uint64_t row_codes8(const float (&v)[8], const RowScale& s) {
  uint32_t b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = row_code(v[j], s.r);
  uint32_t w[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t lo = __builtin_amdgcn_perm(b[4 * j + 1], b[4 * j], 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm(b[4 * j + 3], b[4 * j + 2], 0x04000C0Cu);
    w[j] = lo | hi;
  }
  const uint64_t q = static_cast<uint64_t>(w[1]) << 32 | w[0];
  return s.r > 0.0f ? q : 0u;
}

}  // namespace fgq
