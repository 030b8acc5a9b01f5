// i8gemm.h -- pieces shared by the int8 products with token and channel
// scales: y[m][o] = (sum_k q[m][k] w[o][k]) * sx[m] * sw[o] (+ bias[o]).
//
// Both operands are rows of int8 along k, padded with zeros to a multiple of
// kI8RowStep bytes, so every 128-byte step of k is whole.  Sums are int32
// (K <= kI8MaxK keeps 127 * 128 * K below 2^31); the epilogue converts the
// sum to fp32, multiplies by the two scales one after the other (their
// product could underflow where the result does not) and adds the bias in a
// fused multiply-add: three roundings, then the one to the output's type.
#pragma once

#include "elem.h"
#include "igemm.h"

namespace fgq {
namespace i8 {

struct I8Args {
  const int8_t* q;
  const int8_t* w;
  const float* sx;
  const float* sw;
  const float* bias;  // NULL: none
  void* y;
  int64_t ldq, ldw, ldy;
  int32_t M, O, nk;  // nk: 128-byte steps of k
};

__device__ inline float scaled(int32_t sum, float sx, float sw, float bias) {
  return fmaf(static_cast<float>(sum) * sx, sw, bias);
}

template <int kType>
__device__ inline void put_y(const I8Args& a, int64_t m, int64_t o, float v) {
  if (check_store(kSiteStoreY, m * a.ldy + o, 1, (a.M - 1) * a.ldy + a.O)) Elem<kType>::put(a.y, m * a.ldy + o, v);
}

// Eight consecutive channels of a row (those below O), as wide stores.
template <int kType>
__device__ inline void put8(const I8Args& a, int64_t m, int64_t o, const float (&v)[8]) {
  const int64_t at = m * a.ldy + o;
  if (o + 8 > a.O) {
    for (int c = 0; o + c < a.O; ++c) put_y<kType>(a, m, o + c, v[c]);
  } else if (check_store(kSiteStoreY, at, 8, (a.M - 1) * a.ldy + a.O)) {
    store8<kType>(a.y, at, v);
  }
}

// Tiles of the output, rows by channels (one number: both), times the groups
// of waves that share its k (i8tile.hip).
enum Tile { kTile64x4, kTile64x2, kTile64by128x2, kTile128x2, kTile128, kTile256 };

}  // namespace i8

// Launchers; arguments already validated.
fgq_status launch_i8(const i8::I8Args& a, int32_t y_type, hipStream_t st);
fgq_status launch_i8_tile(const i8::I8Args& a, i8::Tile tile, int32_t y_type, hipStream_t st);
fgq_status launch_i8_few(const i8::I8Args& a, int32_t y_type, hipStream_t st);
// The same on rows that are not yet quantized (a.q and a.sx unused), at most
// 16 of them, whose codes fit in LDS.
fgq_status launch_i8_fused(const void* x, int32_t x_type, int64_t ldx, int64_t K, const i8::I8Args& a, int32_t y_type,
                           hipStream_t st);
// When that is done: up to 8 rows (a wave each), and up to 16 short ones.
// Measured, us (fused, two launches; replayed from a graph, and called one by one,
// where a launch costs the host as much as the kernel takes): 8 rows of 2048,
// O 2048 6.5, 6.8 and 8.3, 12.9; of 4000, O 4096 11.5, 10.6 and 11.3, 13.0; 1 row of
// 4096, O 4096 6.4, 10.1; of 16384, O 8192 31.2, 34.8; 16 rows of 512, O 1024 5.5, 5.2
// and 8.2, 13.2; of 1024, O 4096 7.0, 6.6 and 8.3, 12.9; of 2048, O 8192 12.6, 9.8 and
// 12.3, 12.9.
constexpr bool i8_fused(int64_t M, int64_t row_bytes) {
  return M * (row_bytes + 16) <= (M <= 8 ? 64 << 10 : M <= 16 ? 17 << 10 : 0);
}

}  // namespace fgq
