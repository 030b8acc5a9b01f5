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

}  // namespace i8

// Launchers; arguments already validated.
fgq_status launch_i8_few(const i8::I8Args& a, int32_t y_type, hipStream_t st);

}  // namespace fgq
