// kvattn.hip -- attention over the quantized cache: how a call is divided
// (rows, workgroups, splits of the keys), and the join of split keys.
#include "kvattn.h"

#include <algorithm>

#include "igemm.h"

namespace fgq {
namespace {

constexpr int kJoinThreads = 256;

// One wave a row: the splits' outputs, each divided by nothing yet, weighted
// by 2^(its maximum - the largest), over the sum of the weighted sums.  The
// order of the splits is fixed.
template <int kType>
__global__ __launch_bounds__(kJoinThreads) void kv_attn_join_kernel(KvAttnArgs a) {
  const int lane = threadIdx.x % 64;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * (kJoinThreads / 64) + threadIdx.x / 64;
  if (item >= static_cast<int64_t>(a.B) * a.max_q * a.Hq) return;
  const int head = static_cast<int>(item % a.Hq);
  const int i = static_cast<int>(item / a.Hq % a.max_q), b = static_cast<int>(item / a.Hq / a.max_q);
  const int64_t q0 = max(0, min(a.cu_q[b], static_cast<int>(a.T)));
  const int64_t q1 = max(q0, min(static_cast<int64_t>(a.cu_q[b + 1]), a.T));
  if (i >= q1 - q0) return;
  const int64_t row = (q0 + i) * a.Hq + head;
  const float* p = a.part + row * a.splits * (a.D + 2);
  float mx = -INFINITY;
  for (int s = 0; s < a.splits; ++s) mx = fmaxf(mx, p[s * (a.D + 2) + a.D]);
  const float base = mx == -INFINITY ? 0.0f : mx;
  float sum = 0.0f, v[4] = {0, 0, 0, 0};
  for (int s = 0; s < a.splits; ++s) {
    const float* ps = p + s * (a.D + 2);
    const float w = exp2f(ps[a.D] - base);
    sum += w * ps[a.D + 1];
    for (int j = 0; j < a.D / 64; ++j) v[j] += w * ps[64 * j + lane];
  }
  for (int j = 0; j < a.D / 64; ++j) {
    const int64_t at = row * a.D + 64 * j + lane;
    if (check_store(kSiteStoreY, at, 1, a.T * a.Hq * a.D)) Elem<kType>::put(a.o, at, sum == 0.0f ? 0.0f : v[j] / sum);
  }
  if (lane == 0 && a.lse && check_store(kSiteStoreY, row, 1, a.T * a.Hq))
    a.lse[row] = sum > 0.0f ? (mx + log2f(sum)) * 0.6931471805599453f : (sum == 0.0f ? -INFINITY : sum);
}

struct Plan {
  int nt, tiles, splits, split_keys;
  bool share;
};

Plan plan(int32_t Hq, int32_t Hkv, int64_t B, int64_t max_q, int64_t max_keys) {
  Plan p{};
  const int64_t rows = max_q * (Hq / Hkv);
  p.share = rows <= 64;
  p.nt = rows <= 16 ? 1 : 2;
  p.tiles = static_cast<int>(ceil_div(rows, 16 * p.nt * (p.share ? 1 : 4)));
  p.splits = 1;
  if (p.share) {
    const int64_t wgs = B * Hkv * p.tiles, want = 8LL * ig::device_cus();
    const int64_t most = ceil_div(max_keys, 512);
    p.splits = static_cast<int>(std::max<int64_t>(1, std::min({most, ceil_div(want, wgs), int64_t{256}})));
  }
  p.split_keys = static_cast<int>(round_up(ceil_div(max_keys + 15, p.splits), 512));
  return p;
}

}  // namespace

size_t kv_attn_ws_bytes(int64_t T, int32_t Hq, int32_t Hkv, int32_t D, int64_t B, int64_t max_q, int64_t max_keys) {
  const Plan p = plan(Hq, Hkv, B, max_q, max_keys);
  return p.splits == 1 ? 0 : static_cast<size_t>(T) * Hq * p.splits * (D + 2) * sizeof(float);
}

fgq_status launch_kv_attn(KvAttnArgs a, void* ws, hipStream_t st) {
  const Plan p = plan(a.Hq, a.Hkv, a.B, a.max_q, a.max_pages * a.P);
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.split_keys = p.split_keys;
  a.part = static_cast<float*>(ws);
  const fgq_status rc = a.D == 64    ? launch_kv_attn_d64(a, p.nt, p.share, st)
                        : a.D == 128 ? launch_kv_attn_d128(a, p.nt, p.share, st)
                                     : launch_kv_attn_d256(a, p.nt, p.share, st);
  if (rc != FGQ_OK || p.splits == 1) return rc;
  const int64_t items = static_cast<int64_t>(a.B) * a.max_q * a.Hq;
  const dim3 grid(static_cast<uint32_t>(ceil_div(items, kJoinThreads / 64)));
  if (a.type == FGQ_F16)
    hipLaunchKernelGGL(kv_attn_join_kernel<FGQ_F16>, grid, dim3(kJoinThreads), 0, st, a);
  else
    hipLaunchKernelGGL(kv_attn_join_kernel<FGQ_BF16>, grid, dim3(kJoinThreads), 0, st, a);
  return last_launch();
}

}  // namespace fgq
