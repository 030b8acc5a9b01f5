// rowquant.hip -- fgq_quantize_rows: the rows of a matrix to int8, one scale a
// row.  a = max |x| of the row, scale a / 127, code rint(x * (127 / a)).
//
// The maximum is taken over the absolute values' bit patterns, which order
// like the values and put infinities and NaN above all of them: a row that
// holds one gets the scale NaN and codes 0.  |x * (127 / a)| <= 127 after both
// roundings ((1 + 2^-24)^2 * 127 rounds to 127), so the codes need no clamp.
#include <type_traits>

#include "elem.h"
#include "rowquant.h"

namespace fgq {
namespace {

constexpr int kThreads = 256;

struct RowArgs {
  const void* x;
  int64_t M, K, ldx, ldq;
  int8_t* q;
  float* scale;
};

template <int kType>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(RowArgs a) {
  __shared__ uint32_t red[kThreads / 64];
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const char* x = static_cast<const char*>(a.x) + row * a.ldx * Elem<kType>::kBytes;
  uint32_t m = 0;
  for (int64_t k = 8 * tid; k < a.K; k += 8 * kThreads) {
    if (k + 8 <= a.K) {
      float v[8];
      values8<kType>(load8<kType>(x, k), v);
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, abs_bits(v[j]));
    } else {
      for (int64_t j = k; j < a.K; ++j) m = max(m, abs_bits(Elem<kType>::get(x, j)));
    }
  }
  m = wave_max(m);
  if (tid % 64 == 0) red[tid / 64] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) m = max(m, red[w]);
  const RowScale s = row_scale(m);
  if (tid == 0 && check_store(kSiteStoreQ, row, 1, a.M)) a.scale[row] = s.scale;
  int8_t* q = a.q + row * a.ldq;
  const int64_t Kp = round_up(a.K, kI8RowStep);
  for (int64_t k = 8 * tid; k < Kp; k += 8 * kThreads) {
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (k + 8 <= a.K) {
      values8<kType>(load8<kType>(x, k), v);
    } else {
      for (int j = 0; j < 8; ++j)
        if (k + j < a.K) v[j] = Elem<kType>::get(x, k + j);
    }
    if (check_store(kSiteStoreQ, row * a.ldq + k, 8, a.M * a.ldq))
      *reinterpret_cast<uint64_t*>(q + k) = row_codes8(v, s);
  }
}

}  // namespace

fgq_status launch_quantize_rows(const void* x, int32_t type, int64_t M, int64_t K, int64_t ldx, int8_t* q,
                                int64_t ldq, float* scale, hipStream_t st) {
  const RowArgs a{x, M, K, ldx, ldq, q, scale};
  return with_type(type, [&](auto t) {
    hipLaunchKernelGGL((quantize_rows_kernel<decltype(t)::value>), dim3(static_cast<uint32_t>(M)), dim3(kThreads), 0,
                       st, a);
    return last_launch();
  });
}

}  // namespace fgq
