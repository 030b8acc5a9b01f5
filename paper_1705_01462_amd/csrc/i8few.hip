// i8few.hip -- the int8 product at few rows: a workgroup takes 16 channels
// and 16 kMB rows, its waves share the steps of k and meet in LDS.
//
// The weights are what such a product has to read, and each is read once: a
// lane holds channel l % 16 and, of every 64 k, the 16 at 16 (l / 16), so a
// wave-wide load takes 64 contiguous bytes of 16 rows and goes straight into a
// fragment of the 16x16x64 matrix instruction.  The result has a row of y in
// every lane's column: lane l holds row l % 16, channels 4 (l / 16) + [0, 4).
#include "i8gemm.h"

namespace fgq {
namespace {

using namespace i8;
using ig::v4i;
constexpr int kWaves = 4;

template <int kMB, int kType>
__global__ __launch_bounds__(64 * kWaves) void i8_few_kernel(I8Args a) {
  __shared__ __attribute__((aligned(16))) v4i red[kWaves][kMB * 64];
  const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
  const int g = lane / 16;
  const int n_ot = (a.O + 15) / 16;
  const int o0 = 16 * (blockIdx.x % n_ot);
  const int64_t m0 = static_cast<int64_t>(16 * kMB) * (blockIdx.x / n_ot);
  const int8_t* wp = a.w + min(static_cast<int64_t>(o0 + lane % 16), static_cast<int64_t>(a.O) - 1) * a.ldw + 16 * g;
  const int8_t* qp[kMB];
#pragma unroll
  for (int b = 0; b < kMB; ++b)
    qp[b] = a.q + min(m0 + 16 * b + lane % 16, static_cast<int64_t>(a.M) - 1) * a.ldq + 16 * g;
  v4i acc[kMB];
#pragma unroll
  for (int b = 0; b < kMB; ++b) acc[b] = v4i{0, 0, 0, 0};
  for (int s = wave; s < 2 * a.nk; s += kWaves) {
    const v4i wf = *reinterpret_cast<const v4i*>(wp + 64 * static_cast<int64_t>(s));
#pragma unroll
    for (int b = 0; b < kMB; ++b) {
      const v4i xf = *reinterpret_cast<const v4i*>(qp[b] + 64 * static_cast<int64_t>(s));
      acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, xf, acc[b], 0, 0, 0);
    }
  }
#pragma unroll
  for (int b = 0; b < kMB; ++b) red[wave][64 * b + lane] = acc[b];
  __syncthreads();
  for (int b = wave; b < kMB; b += kWaves) {
    v4i S = red[0][64 * b + lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) S += red[w][64 * b + lane];
    const int64_t m = m0 + 16 * b + lane % 16;
    if (m >= a.M) continue;
    const float sx = a.sx[m];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int o = o0 + 4 * g + c;
      if (o < a.O) put_y<kType>(a, m, o, scaled(S[c], sx, a.sw[o], a.bias ? a.bias[o] : 0.0f));
    }
  }
}

}  // namespace

fgq_status launch_i8_few(const I8Args& a, int32_t y_type, hipStream_t st) {
  return with_type(y_type, [&](auto t) {
    constexpr int kMB = 4;
    const dim3 grid(static_cast<uint32_t>(ceil_div(a.O, 16) * ceil_div(a.M, 16 * kMB)));
    hipLaunchKernelGGL((i8_few_kernel<kMB, decltype(t)::value>), grid, dim3(64 * kWaves), 0, st, a);
    return last_launch();
  });
}

}  // namespace fgq
